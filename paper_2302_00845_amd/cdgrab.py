"""ctypes binding of libcdgrab.so: argument marshalling only.

Every function takes torch tensors that already live on the GPU, checks their
dtype / shape / contiguity, and passes raw device pointers through the C ABI.
There is no fallback: if the shared library is missing, loading raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch  # loaded first so that the HIP runtime torch ships is the one in the process

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libcdgrab.so")
_lib = None

CDGRAB_OK, CDGRAB_EINVAL, CDGRAB_ENOMEM, CDGRAB_EHIP, CDGRAB_EGEN = 0, -1, -2, -3, -4

GEN_FN = ctypes.CFUNCTYPE(ctypes.c_int, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64,
                          ctypes.c_void_p, ctypes.c_void_p)


class CdgrabError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__("cdgrab error %d: %s" % (code, text))
        self.code = code


class _Options(ctypes.Structure):
    _fields_ = [("device", ctypes.c_int32), ("block_pairs", ctypes.c_int32),
                ("stream", ctypes.c_void_p), ("timing", ctypes.c_int32),
                ("pass1_groups", ctypes.c_int32), ("apply_mode", ctypes.c_int32),
                ("gram_mode", ctypes.c_int32), ("apply_groups", ctypes.c_int32)]


class Timing(ctypes.Structure):
    _fields_ = [("generator_ms", ctypes.c_double), ("balance_ms", ctypes.c_double),
                ("pass1_ms", ctypes.c_double), ("reduce_ms", ctypes.c_double),
                ("resolve_ms", ctypes.c_double), ("pass2_ms", ctypes.c_double),
                ("finish_ms", ctypes.c_double), ("blocks", ctypes.c_int64),
                ("block_pairs", ctypes.c_int32), ("pass1_groups", ctypes.c_int32)]

    def as_dict(self):
        return {name: getattr(self, name) for name, _ in self._fields_}


class Plan(ctypes.Structure):
    _fields_ = [("pairs", ctypes.c_int64), ("blocks", ctypes.c_int64),
                ("block_pairs", ctypes.c_int32), ("vector_width", ctypes.c_int32),
                ("tile_elems", ctypes.c_int32), ("fused_apply", ctypes.c_int32),
                ("pass1_groups", ctypes.c_int32), ("pass2_groups", ctypes.c_int32),
                ("gram_ahead", ctypes.c_int32), ("step_pairs", ctypes.c_int32),
                ("workspace_bytes", ctypes.c_int64), ("staging_bytes", ctypes.c_int64),
                ("bytes_per_example", ctypes.c_double)]

    def as_dict(self):
        return {name: getattr(self, name) for name, _ in self._fields_}


class _TokenRows(ctypes.Structure):
    _fields_ = [("examples", ctypes.c_int64), ("rows", ctypes.c_int64), ("tokens", ctypes.c_int64),
                ("first", ctypes.c_void_p), ("count", ctypes.c_void_p)]


class _Heads(ctypes.Structure):
    _fields_ = [("q_heads", ctypes.c_int64), ("k_heads", ctypes.c_int64), ("dim", ctypes.c_int64),
                ("base", ctypes.c_double), ("eps", ctypes.c_float)]


_ELEM = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}  # CDGRAB_F32, _BF16, _F16


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Load libcdgrab.so (built by ``python -m paper_2302_00845_amd.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise FileNotFoundError(
            "%s is missing: build it with `python -m paper_2302_00845_amd.build` "
            "(there is no fallback path)" % _LIB_PATH)
    lib = ctypes.CDLL(_LIB_PATH)
    P, i64, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
    lib.cdgrab_create.argtypes = [ctypes.POINTER(P), ctypes.POINTER(_Options)]
    lib.cdgrab_create.restype = ctypes.c_int
    lib.cdgrab_destroy.argtypes = [P]
    lib.cdgrab_destroy.restype = ctypes.c_int
    lib.cdgrab_last_error.argtypes = [P]
    lib.cdgrab_last_error.restype = ctypes.c_char_p
    lib.cdgrab_plan_epoch.argtypes = [i64, i64, i64, i32, i32, i64, ctypes.POINTER(Plan)]
    lib.cdgrab_plan_epoch.restype = ctypes.c_int
    lib.cdgrab_pergrad.argtypes = [P, i64, i64, i64, P, P, P, P]
    lib.cdgrab_pergrad.restype = ctypes.c_int
    lib.cdgrab_balance_epoch.argtypes = [P, i64, i64, i64, P, P, P, P, P, P, P, P, P]
    lib.cdgrab_balance_epoch.restype = ctypes.c_int
    lib.cdgrab_reorder.argtypes = [P, i64, i64, P, P, P]
    lib.cdgrab_reorder.restype = ctypes.c_int
    lib.cdgrab_balance_epoch_randomized.argtypes = [P, i64, i64, i64, P, P, P, P, P, P, P]
    lib.cdgrab_balance_epoch_randomized.restype = ctypes.c_int
    lib.cdgrab_balance_epoch_stale_mean.argtypes = [P, i64, i64, P, P, P, P, P, P, P]
    lib.cdgrab_balance_epoch_stale_mean.restype = ctypes.c_int
    lib.cdgrab_balance_epoch_independent.argtypes = [P, i64, i64, i64, P, P, P, P]
    lib.cdgrab_balance_epoch_independent.restype = ctypes.c_int
    lib.cdgrab_train_epoch_softmax.argtypes = [P, i64, i64, i64, i64, P, P, P, P, P, ctypes.c_float,
                                               ctypes.c_float, P, P, P, P]
    lib.cdgrab_train_epoch_softmax.restype = ctypes.c_int
    lib.cdgrab_train_softmax.argtypes = [P, i64, i64, i64, i64, P, P, P, P, P, ctypes.c_float,
                                         ctypes.c_float, i64, P, P]
    lib.cdgrab_train_softmax.restype = ctypes.c_int
    lib.cdgrab_herding_bound.argtypes = [P, i64, i64, i64, P, P, P]
    lib.cdgrab_herding_bound.restype = ctypes.c_int
    lib.cdgrab_balance_epoch_static.argtypes = [P, i64, i64, i64, P, P, P, P, P, P, P]
    lib.cdgrab_balance_epoch_static.restype = ctypes.c_int
    lib.cdgrab_train_epoch_softmax_orthogonal.argtypes = [P, i64, i64, i64, i64, P, P, P, P, P, ctypes.c_float,
                                                          ctypes.c_float, i32, P, P, P, P, P]
    lib.cdgrab_train_epoch_softmax_orthogonal.restype = ctypes.c_int
    lib.cdgrab_layernorm.argtypes = [P, i64, i64, i32, P, i64, P, P, ctypes.c_float, P, i64]
    lib.cdgrab_layernorm.restype = ctypes.c_int
    lib.cdgrab_pergrad_layernorm.argtypes = [P, ctypes.POINTER(_TokenRows), i64, i32, P, i64, P, i64, P,
                                             ctypes.c_float, P, i64, i32, P, i64]
    lib.cdgrab_pergrad_layernorm.restype = ctypes.c_int
    lib.cdgrab_pergrad_linear.argtypes = [P, ctypes.POINTER(_TokenRows), i64, i64, i32, P, i64, P, i64, i32, P, i64]
    lib.cdgrab_pergrad_linear.restype = ctypes.c_int
    lib.cdgrab_orthogonalize.argtypes = [P, i64, i64, i64, i32, P, i64, i64, i32, P, P, i64, i64]
    lib.cdgrab_orthogonalize.restype = ctypes.c_int
    f32, rows_of, heads_of = ctypes.c_float, ctypes.POINTER(_TokenRows), ctypes.POINTER(_Heads)
    lib.cdgrab_embed.argtypes = [P, i64, i64, i64, P, i32, P, i64, f32, i32, P, i64]
    lib.cdgrab_embed.restype = ctypes.c_int
    lib.cdgrab_pergrad_embed.argtypes = [P, rows_of, i64, i64, i32, P, P, i64, f32, P, i64]
    lib.cdgrab_pergrad_embed.restype = ctypes.c_int
    lib.cdgrab_headnorm.argtypes = [P, rows_of, heads_of, i32, P, i64, P, P, P, i64]
    lib.cdgrab_headnorm.restype = ctypes.c_int
    lib.cdgrab_pergrad_headnorm.argtypes = [P, rows_of, heads_of, i32, P, i64, P, i64, P, P, P, i64, P, i64]
    lib.cdgrab_pergrad_headnorm.restype = ctypes.c_int
    lib.cdgrab_attention.argtypes = [P, rows_of, i64, i64, i64, i32, f32] + [P, i64] * 4 + [P]
    lib.cdgrab_attention.restype = ctypes.c_int
    lib.cdgrab_attention_backward.argtypes = [P, rows_of, i64, i64, i64, i32, f32] + [P, i64] * 4 + [P] + [P, i64] * 4
    lib.cdgrab_attention_backward.restype = ctypes.c_int
    lib.cdgrab_get_timing.argtypes = [P, ctypes.POINTER(Timing)]
    lib.cdgrab_get_timing.restype = ctypes.c_int
    _lib = lib
    return lib


def cdgrab_plan_epoch(m: int, n: int, d: int, block_pairs: int = 0, streamed: bool = False,
                      base_align: int = 16) -> dict:
    """Host-only blocking plan (cdgrab_plan_epoch)."""
    lib = load_library()
    plan = Plan()
    rc = lib.cdgrab_plan_epoch(m, n, d, block_pairs, 1 if streamed else 0, base_align,
                               ctypes.byref(plan))
    if rc != CDGRAB_OK:
        raise CdgrabError(rc, "cdgrab_plan_epoch rejected m=%d n=%d d=%d block_pairs=%d" % (m, n, d, block_pairs))
    return plan.as_dict()


def _ptr(t: Optional[torch.Tensor], dtype, shape, name, device) -> Optional[int]:
    if t is None:
        return None
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if tuple(t.shape) != tuple(shape):
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if t.device != device:
        raise ValueError("%s must live on %s, got %s" % (name, device, t.device))
    return t.data_ptr()


# The current stream's number (torch.cuda.current_stream makes an object of it: 2 us, a third of a small call).
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _allocator(h):
    """torch.empty for the outputs of a call.  They are allocated on the handle's stream, where the call writes them: memory
    that the current stream has let go of may still be in use there.  The current stream is taken to be where they will be
    read."""
    if h.stream is None or h.stream_number == _current_stream(h.device_index):
        return torch.empty

    def empty(shape, **kinds):
        with torch.cuda.stream(h.stream):
            out = torch.empty(shape, **kinds)
        out.record_stream(torch.cuda.current_stream(h.device))
        return out
    return empty


def _empty_like(h, t: torch.Tensor) -> torch.Tensor:
    if h.stream is None or h.stream_number == _current_stream(h.device_index):
        return torch.empty_like(t, memory_format=torch.contiguous_format)
    return _allocator(h)(t.shape, dtype=t.dtype, device=t.device)


class Handle:
    """Owns a cdgrab_handle (workspace + stream binding) on one GPU.

    Calls run on the handle's stream.  Where that is not the current stream, the caller orders the inputs before the call and
    what reads the outputs after it, as between any two streams."""

    def __init__(self, device: int = 0, block_pairs: int = 0, timing: int = 0,
                 pass1_groups: int = 0, stream: Optional[torch.cuda.Stream] = None,
                 apply_mode: int = 0, gram_mode: int = 0, apply_groups: int = 0):
        self._lib = load_library()
        self.device = torch.device("cuda", device)
        if stream is None:
            stream = torch.cuda.current_stream(self.device)
        self.stream = stream
        self.stream_number, self.device_index = stream.cuda_stream, device
        opt = _Options(device=device, block_pairs=block_pairs, stream=stream.cuda_stream,
                       timing=timing, pass1_groups=pass1_groups,
                       apply_mode=apply_mode, gram_mode=gram_mode, apply_groups=apply_groups)
        h = ctypes.c_void_p()
        rc = self._lib.cdgrab_create(ctypes.byref(h), ctypes.byref(opt))
        if rc != CDGRAB_OK:
            raise CdgrabError(rc, self._lib.cdgrab_last_error(None).decode())
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            self._lib.cdgrab_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc: int):
        if rc != CDGRAB_OK:
            raise CdgrabError(rc, self._lib.cdgrab_last_error(self._h).decode())

    def timing(self) -> dict:
        t = Timing()
        self._check(self._lib.cdgrab_get_timing(self._h, ctypes.byref(t)))
        return t.as_dict()


def cdgrab_pergrad(h: Handle, X: torch.Tensor, y: torch.Tensor, W: torch.Tensor,
                   G_out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Per-example softmax cross-entropy gradients G[N][(in_dim+1)*classes]."""
    N, in_dim = X.shape
    classes = W.shape[1]
    if G_out is None:
        G_out = _allocator(h)((N, (in_dim + 1) * classes), dtype=torch.float32, device=h.device)
    h._check(h._lib.cdgrab_pergrad(
        h._h, N, in_dim, classes,
        _ptr(X, torch.float32, (N, in_dim), "X", h.device),
        _ptr(y, torch.int32, (N,), "y", h.device),
        _ptr(W, torch.float32, (in_dim + 1, classes), "W", h.device),
        _ptr(G_out, torch.float32, (N, (in_dim + 1) * classes), "G_out", h.device)))
    return G_out


def cdgrab_balance_epoch(h: Handle, m: int, n: int, d: int,
                         grads: Optional[torch.Tensor] = None,
                         gen=None, gen_ctx: Optional[int] = None,
                         perm_in: Optional[torch.Tensor] = None,
                         want_r32: bool = True, want_r64: bool = False,
                         want_dots: bool = False) -> dict:
    """One epoch of coordinated pair balancing.

    ``grads`` is a [m][n][d] fp32 GPU tensor, or ``gen`` is a C function pointer
    (cdgrab_gen_fn, e.g. taken from another shared library with ctypes) with its
    context pointer ``gen_ctx``.  Returns the output tensors in a dict.
    """
    dev = h.device
    half = n // 2 if n >= 0 else 0
    empty = _allocator(h)
    signs = empty((max(m, 0), max(half, 0)), dtype=torch.int8, device=dev)
    perm = empty((max(m, 0), max(n, 0)), dtype=torch.int32, device=dev)
    r32 = empty((max(d, 0),), dtype=torch.float32, device=dev) if want_r32 else None
    r64 = empty((max(d, 0),), dtype=torch.float64, device=dev) if want_r64 else None
    dots = empty((max(m, 0), max(half, 0)), dtype=torch.float64, device=dev) if want_dots else None
    gptr = _ptr(grads, torch.float32, (m, n, d), "grads", dev) if grads is not None else None
    gen_ptr = ctypes.cast(gen, ctypes.c_void_p) if gen is not None else None
    h._check(h._lib.cdgrab_balance_epoch(
        h._h, m, n, d, gptr, gen_ptr, gen_ctx,
        _ptr(perm_in, torch.int32, (m, n), "perm_in", dev),
        signs.data_ptr(), perm.data_ptr(),
        r32.data_ptr() if r32 is not None else None,
        r64.data_ptr() if r64 is not None else None,
        dots.data_ptr() if dots is not None else None))
    return {"signs": signs, "perm": perm, "r32": r32, "r64": r64, "dots": dots}


def cdgrab_balance_epoch_static(h: Handle, grads: torch.Tensor, out: dict,
                                perm_in: Optional[torch.Tensor] = None) -> dict:
    """cdgrab_balance_epoch on the library's static workspace (dense input, rows of at most
    CDGRAB_STATIC_MAX_D elements).  The call allocates nothing: ``out`` holds the caller's
    output tensors ``signs`` [m][n/2] int8 and ``perm`` [m][n] int32, and optionally ``r32``
    [d] float32, ``r64`` [d] float64, ``dots`` [m][n/2] float64."""
    m, n, d = grads.shape
    dev = h.device
    h._check(h._lib.cdgrab_balance_epoch_static(
        h._h, m, n, d, _ptr(grads, torch.float32, (m, n, d), "grads", dev),
        _ptr(perm_in, torch.int32, (m, n), "perm_in", dev),
        _ptr(out["signs"], torch.int8, (m, n // 2), "signs", dev),
        _ptr(out["perm"], torch.int32, (m, n), "perm", dev),
        _ptr(out.get("r32"), torch.float32, (d,), "r32", dev),
        _ptr(out.get("r64"), torch.float64, (d,), "r64", dev),
        _ptr(out.get("dots"), torch.float64, (m, n // 2), "dots", dev)))
    return out


def cdgrab_reorder(h: Handle, signs: torch.Tensor, perm_in: Optional[torch.Tensor] = None) -> torch.Tensor:
    """General reorder from per-example +-1 signs [m][n] (int8)."""
    m, n = signs.shape
    out = _allocator(h)((m, n), dtype=torch.int32, device=h.device)
    h._check(h._lib.cdgrab_reorder(
        h._h, m, n, _ptr(signs, torch.int8, (m, n), "signs", h.device),
        _ptr(perm_in, torch.int32, (m, n), "perm_in", h.device), out.data_ptr()))
    return out


def cdgrab_herding_bound(h: Handle, z: torch.Tensor, perm: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Parallel herding objective of z[m][n][d] (indexed by example id) visited in
    the orders perm[m][n]; returns a one-element float64 GPU tensor."""
    m, n, d = z.shape
    out = _allocator(h)((1,), dtype=torch.float64, device=h.device)
    h._check(h._lib.cdgrab_herding_bound(
        h._h, m, n, d, _ptr(z, torch.float32, (m, n, d), "z", h.device),
        _ptr(perm, torch.int32, (m, n), "perm", h.device), out.data_ptr()))
    return out


def cdgrab_train_epoch_softmax(h: Handle, X: torch.Tensor, y: torch.Tensor, W: torch.Tensor,
                               perm_in: Optional[torch.Tensor] = None,
                               velocity: Optional[torch.Tensor] = None, lr: float = 0.1,
                               momentum: float = 0.0, want_grads: bool = False,
                               want_loss: bool = True) -> dict:
    """One CD-GraB training epoch of the softmax-regression model; W (and velocity)
    are updated in place.  X[m][n][in_dim], y[m][n]."""
    m, n, in_dim = X.shape
    classes = W.shape[1]
    d = (in_dim + 1) * classes
    dev = h.device
    empty = _allocator(h)
    signs = empty((m, n // 2), dtype=torch.int8, device=dev)
    perm = empty((m, n), dtype=torch.int32, device=dev)
    grads = empty((m, n, d), dtype=torch.float32, device=dev) if want_grads else None
    loss = empty((m, n), dtype=torch.float32, device=dev) if want_loss else None
    h._check(h._lib.cdgrab_train_epoch_softmax(
        h._h, m, n, in_dim, classes,
        _ptr(X, torch.float32, (m, n, in_dim), "X", dev), _ptr(y, torch.int32, (m, n), "y", dev),
        _ptr(perm_in, torch.int32, (m, n), "perm_in", dev),
        _ptr(W, torch.float32, (in_dim + 1, classes), "W", dev),
        _ptr(velocity, torch.float32, (d,), "velocity", dev), lr, momentum,
        signs.data_ptr(), perm.data_ptr(),
        grads.data_ptr() if grads is not None else None,
        loss.data_ptr() if loss is not None else None))
    return {"signs": signs, "perm": perm, "grads": grads, "loss": loss}


def cdgrab_train_softmax(h: Handle, X: torch.Tensor, y: torch.Tensor, W: torch.Tensor,
                         perm: torch.Tensor, epochs: int,
                         velocity: Optional[torch.Tensor] = None, lr: float = 0.1,
                         momentum: float = 0.0, want_loss: bool = True) -> dict:
    """`epochs` CD-GraB training epochs with the permutations carried over; W, velocity
    and perm[m][n] (first order in, next order out) are updated in place."""
    m, n, in_dim = X.shape
    classes = W.shape[1]
    d = (in_dim + 1) * classes
    dev = h.device
    empty = _allocator(h)
    signs = empty((m, n // 2), dtype=torch.int8, device=dev)
    loss = empty((epochs, m, n), dtype=torch.float32, device=dev) if want_loss else None
    h._check(h._lib.cdgrab_train_softmax(
        h._h, m, n, in_dim, classes,
        _ptr(X, torch.float32, (m, n, in_dim), "X", dev), _ptr(y, torch.int32, (m, n), "y", dev),
        _ptr(perm, torch.int32, (m, n), "perm", dev),
        _ptr(W, torch.float32, (in_dim + 1, classes), "W", dev),
        _ptr(velocity, torch.float32, (d,), "velocity", dev), lr, momentum, epochs,
        signs.data_ptr(), loss.data_ptr() if loss is not None else None))
    return {"signs": signs, "perm": perm, "loss": loss}


def cdgrab_balance_epoch_independent(h: Handle, grads: torch.Tensor,
                                     perm_in: Optional[torch.Tensor] = None) -> dict:
    """ID-GraB (PairBal): m independent one-worker walks over grads[m][n][d]."""
    m, n, d = grads.shape
    empty = _allocator(h)
    signs = empty((m, n // 2), dtype=torch.int8, device=h.device)
    perm = empty((m, n), dtype=torch.int32, device=h.device)
    h._check(h._lib.cdgrab_balance_epoch_independent(
        h._h, m, n, d, _ptr(grads, torch.float32, (m, n, d), "grads", h.device),
        _ptr(perm_in, torch.int32, (m, n), "perm_in", h.device), signs.data_ptr(), perm.data_ptr()))
    return {"signs": signs, "perm": perm}


def cdgrab_balance_epoch_stale_mean(h: Handle, grads: torch.Tensor,
                                    stale_mean: Optional[torch.Tensor] = None,
                                    perm_in: Optional[torch.Tensor] = None) -> dict:
    """Centralized GraB balancing of grads[n][d] centred by a stale mean."""
    n, d = grads.shape
    dev = h.device
    empty = _allocator(h)
    signs = empty((n,), dtype=torch.int8, device=dev)
    perm = empty((n,), dtype=torch.int32, device=dev)
    mean = empty((d,), dtype=torch.float32, device=dev)
    r64 = empty((d,), dtype=torch.float64, device=dev)
    h._check(h._lib.cdgrab_balance_epoch_stale_mean(
        h._h, n, d, _ptr(grads, torch.float32, (n, d), "grads", dev),
        _ptr(stale_mean, torch.float32, (d,), "stale_mean", dev),
        _ptr(perm_in, torch.int32, (n,), "perm_in", dev),
        signs.data_ptr(), perm.data_ptr(), mean.data_ptr(), r64.data_ptr()))
    return {"signs": signs, "perm": perm, "mean": mean, "r64": r64}


def cdgrab_balance_epoch_randomized(h: Handle, grads: torch.Tensor, uniforms: torch.Tensor,
                                    perm_in: Optional[torch.Tensor] = None) -> dict:
    """cdgrab_balance_epoch with the randomized sign rule; uniforms[m][n/2] in [0,1)."""
    m, n, d = grads.shape
    dev = h.device
    empty = _allocator(h)
    signs = empty((m, n // 2), dtype=torch.int8, device=dev)
    perm = empty((m, n), dtype=torch.int32, device=dev)
    r64 = empty((d,), dtype=torch.float64, device=dev)
    dots = empty((m, n // 2), dtype=torch.float64, device=dev)
    h._check(h._lib.cdgrab_balance_epoch_randomized(
        h._h, m, n, d, _ptr(grads, torch.float32, (m, n, d), "grads", dev),
        _ptr(uniforms, torch.float32, (m, n // 2), "uniforms", dev),
        _ptr(perm_in, torch.int32, (m, n), "perm_in", dev),
        signs.data_ptr(), perm.data_ptr(), r64.data_ptr(), dots.data_ptr()))
    return {"signs": signs, "perm": perm, "r64": r64, "dots": dots}


# ---- per-example gradients of layers --------------------------------------------------------

def _rows(t: torch.Tensor, name: str, device, like: Optional[torch.Tensor] = None):
    """(pointer, rows, width, stride) of an array of rows: [..., width] with elements side by side and one
    distance from row to row.  `like`: of the same type and shape."""
    if t.dtype not in _ELEM:
        raise TypeError("%s must be float32, bfloat16 or float16, got %s" % (name, t.dtype))
    if t.device != device:
        raise ValueError("%s must live on %s, got %s" % (name, device, t.device))
    shape = t.shape
    if like is not None and (shape != like.shape or t.dtype != like.dtype):
        raise ValueError("%s must be %s %s, got %s %s" % (name, like.dtype, tuple(like.shape), t.dtype, tuple(shape)))
    if len(shape) < 2:
        raise ValueError("%s must have rows and a width, got shape %s" % (name, tuple(shape)))
    width = shape[-1]
    if t.is_contiguous():
        return t.data_ptr(), t.numel() // width if width else 0, width, width or 1
    strides = t.stride()
    if len(shape) == 3 and strides[2] == 1 and strides[1] >= width > 0 and strides[0] == shape[1] * strides[1] > 0 < shape[0]:
        return t.data_ptr(), shape[0] * shape[1], width, strides[1]  # (the usual case, without the loops)
    rows, stride = 1, width
    for n in shape[:-1]:
        rows *= n
    if rows and width:
        if t.stride(-1) != 1 and width > 1:
            raise ValueError("%s: the elements of a row must lie side by side" % name)
        steps = [(n, s) for n, s in zip(shape[:-1], t.stride()[:-1]) if n > 1]
        if steps:
            stride = steps[-1][1]
            for (_, outer), (n, inner) in zip(steps, steps[1:]):
                if outer != n * inner:
                    raise ValueError("%s: rows must be one distance apart" % name)
            if stride < width:
                raise ValueError("%s: rows must not overlap" % name)
    return t.data_ptr(), rows, width, max(stride, 1)


def _vector(t: Optional[torch.Tensor], n: int, name: str, device) -> Optional[int]:
    """Pointer of a contiguous float32 [n], or None."""
    if t is None:
        return None
    if t.dtype is torch.float32 and t.dim() == 1 and t.shape[0] == n and t.is_contiguous() and t.device == device:
        return t.data_ptr()
    return _ptr(t, torch.float32, (n,), name, device)  # (says what is wrong)


def _token_rows(X: torch.Tensor, rows: int, first, count, tokens: Optional[int], device) -> _TokenRows:
    """X is [examples][tokens][width], or [rows][width] with `first` and `tokens` (packed)."""
    if first is None:
        if X.dim() != 3:
            raise ValueError("X must be [examples][tokens][width] unless `first` says where examples start")
        examples, own, _ = X.shape
        if tokens is not None and tokens != own:
            raise ValueError("tokens is %d, and X has %d per example" % (tokens, own))
        tokens = own
        if count is None:
            return _TokenRows(examples, rows, tokens, None, None)
    else:
        if tokens is None:
            raise ValueError("`first` needs `tokens`, the rows that an example has at most")
        examples = first.shape[0] if first.dim() == 1 else -1
    return _TokenRows(examples, rows, tokens, _ptr(first, torch.int64, (examples,), "first", device),
                      _ptr(count, torch.int32, (examples,), "count", device))


def _grad_rows(h, G_out: Optional[torch.Tensor], examples: int, d: int):
    """(G, stride): [examples][d] fp32, a stretch of longer rows if given so."""
    if G_out is None:
        return _allocator(h)((examples, d), dtype=torch.float32, device=h.device), d or 1
    if G_out.dtype != torch.float32:
        raise TypeError("G_out must be float32, got %s" % G_out.dtype)
    if tuple(G_out.shape) != (examples, d):
        raise ValueError("G_out must have shape %s, got %s" % ((examples, d), tuple(G_out.shape)))
    _, _, _, stride = _rows(G_out, "G_out", h.device)
    return G_out, stride


def cdgrab_layernorm(h: Handle, X: torch.Tensor, gain: Optional[torch.Tensor] = None,
                     bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
                     Y: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Layer norm over the last axis of X[..., width]; gain and bias [width] float32."""
    dev = h.device
    px, rows, width, sx = _rows(X, "X", dev)
    if Y is None:
        Y = _empty_like(h, X)
        py, sy = Y.data_ptr(), width or 1
    else:
        py, _, _, sy = _rows(Y, "Y", dev, X)
    rc = h._lib.cdgrab_layernorm(h._h, rows, width, _ELEM[X.dtype], px, sx, _vector(gain, width, "gain", dev),
                                 _vector(bias, width, "bias", dev), eps, py, sy)
    if rc:
        h._check(rc)
    return Y


def cdgrab_pergrad_layernorm(h: Handle, X: torch.Tensor, dY: torch.Tensor, gain: Optional[torch.Tensor] = None,
                             eps: float = 1e-5, first: Optional[torch.Tensor] = None,
                             count: Optional[torch.Tensor] = None, tokens: Optional[int] = None,
                             dX: Optional[torch.Tensor] = None, G_out: Optional[torch.Tensor] = None,
                             with_bias: bool = True, want_dx: bool = True, want_grads: bool = True):
    """Backward pass of cdgrab_layernorm: (dX, G), G[examples][gain's gradient | bias's gradient].

    X and dY are [examples][tokens][width] (with `count` a padded batch), or [rows][width] with the examples' rows
    packed: `first` [examples] int64, `count` int32, `tokens` at most.  Rows of no example keep what dX holds (zero
    where the call makes dX).  G_out may be a stretch of columns of longer rows."""
    dev = h.device
    px, rows, width, sx = _rows(X, "X", dev)
    py, _, _, sy = _rows(dY, "dY", dev, X)
    t = _token_rows(X, rows, first, count, tokens, dev)
    pd, sd = None, width
    if dX is not None:
        pd, _, _, sd = _rows(dX, "dX", dev, X)
    elif want_dx:
        dX = _empty_like(h, X)
        if first is not None or count is not None:
            with torch.cuda.stream(h.stream):  # before the call's kernels, wherever they run
                dX.zero_()
        pd, sd = dX.data_ptr(), width or 1
    G, pg, sg = None, None, 0
    if G_out is not None or want_grads:
        G, sg = _grad_rows(h, G_out, t.examples, (2 if with_bias else 1) * width)
        pg = G.data_ptr()
    rc = h._lib.cdgrab_pergrad_layernorm(h._h, ctypes.byref(t), width, _ELEM[X.dtype], px, sx, py, sy,
                                         _vector(gain, width, "gain", dev), eps, pd, sd, 1 if with_bias else 0, pg, sg)
    if rc:
        h._check(rc)
    return dX, G


def cdgrab_pergrad_linear(h: Handle, X: torch.Tensor, D: torch.Tensor, with_bias: bool = True,
                          first: Optional[torch.Tensor] = None, count: Optional[torch.Tensor] = None,
                          tokens: Optional[int] = None, G_out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Per-example gradients G[examples][(in + 1) * out] of a linear layer's weights (last `out`: the bias) from its
    inputs X and its outputs' gradients D; rows of examples as in cdgrab_pergrad_layernorm."""
    dev = h.device
    px, rows, n_in, sx = _rows(X, "X", dev)
    pd, _, n_out, sd = _rows(D, "D", dev)
    if D.dtype != X.dtype or D.shape[:-1] != X.shape[:-1]:
        raise ValueError("D must be %s of rows %s, got %s %s" % (X.dtype, tuple(X.shape[:-1]), D.dtype, tuple(D.shape)))
    t = _token_rows(X, rows, first, count, tokens, dev)
    G, sg = _grad_rows(h, G_out, t.examples, (n_in + (1 if with_bias else 0)) * n_out)
    rc = h._lib.cdgrab_pergrad_linear(h._h, ctypes.byref(t), n_in, n_out, _ELEM[X.dtype], px, sx, pd, sd,
                                      1 if with_bias else 0, G.data_ptr(), sg)
    if rc:
        h._check(rc)
    return G


def _coeffs(coeffs):
    if coeffs is None:
        return None
    a, b, c = (float(v) for v in coeffs)
    return (ctypes.c_double * 3)(a, b, c)


def cdgrab_orthogonalize(h: Handle, M: torch.Tensor, steps: int = 5, coeffs=None,
                         out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """M[rows][cols] or [batch][rows][cols] with its singular values brought near one (Newton-Schulz products;
    coeffs (a, b, c) of a x + b x^3 + c x^5)."""
    if M.dim() not in (2, 3):
        raise ValueError("M must be [rows][cols] or [batch][rows][cols], got %s" % (tuple(M.shape),))
    if out is None:
        out = _empty_like(h, M)
    elif out.dtype != M.dtype or out.shape != M.shape:
        raise ValueError("out must be %s %s, got %s %s" % (M.dtype, tuple(M.shape), out.dtype, tuple(out.shape)))
    if M.dtype not in _ELEM:
        raise TypeError("M must be float32, bfloat16 or float16, got %s" % M.dtype)
    rows, cols = M.shape[-2:]
    at = []
    for t, name in ((M, "M"), (out, "out")):
        if t.device != h.device:
            raise ValueError("%s must live on %s, got %s" % (name, h.device, t.device))
        strides = t.stride()
        if cols > 1 and strides[-1] != 1:
            raise ValueError("%s: the elements of a row must lie side by side" % name)
        at.append((t.data_ptr(), strides[-2] if rows > 1 else cols, strides[0]))
    rc = h._lib.cdgrab_orthogonalize(h._h, M.shape[0] if M.dim() == 3 else 1, rows, cols, _ELEM[M.dtype], *at[0], steps,
                                     _coeffs(coeffs), *at[1])
    if rc:
        h._check(rc)
    return out


# ---- operators over the rows of a sequence ---------------------------------------------------

def _ids(ids: torch.Tensor, shape, device) -> int:
    if ids.dtype is torch.int32 and ids.shape == shape and ids.is_contiguous() and ids.device == device:
        return ids.data_ptr()
    return _ptr(ids, torch.int32, shape, "ids", device)  # (says what is wrong)


def _made_like(h, t: torch.Tensor, shape, dtype, partly: bool) -> torch.Tensor:
    """An output that the call makes; zeros where it may not write all of it (`partly`)."""
    if h.stream is None or h.stream_number == _current_stream(h.device_index):
        return (torch.zeros if partly else torch.empty)(shape, dtype=dtype, device=t.device)
    out = _allocator(h)(shape, dtype=dtype, device=t.device)
    if partly:
        with torch.cuda.stream(h.stream):  # before the call's kernels, wherever they run
            out.zero_()
    return out


def cdgrab_embed(h: Handle, ids: torch.Tensor, table: torch.Tensor, scale: float = 1.0,
                 dtype: Optional[torch.dtype] = None, Y: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Y[..., width] = scale * table[ids], ids [...] int32, table [vocab][width] float32 or of Y's type (``dtype``, by
    default the table's); zeros for an id outside the table."""
    dev = h.device
    pt, vocab, width, st = _rows(table, "table", dev)
    if table.dim() != 2:
        raise ValueError("table must be [vocab][width], got %s" % (tuple(table.shape),))
    rows = ids.numel()
    if Y is None:
        Y = _made_like(h, table, (*ids.shape, width), dtype or table.dtype, False)
        py, sy = Y.data_ptr(), width or 1
    elif tuple(Y.shape) != (*ids.shape, width) or (dtype is not None and Y.dtype != dtype):
        raise ValueError("Y must be %s %s, got %s %s" % (dtype or table.dtype, (*ids.shape, width), Y.dtype, tuple(Y.shape)))
    else:
        py, _, _, sy = _rows(Y if Y.dim() > 1 else Y.unsqueeze(0), "Y", dev)
    if Y.dtype not in _ELEM:
        raise TypeError("Y must be float32, bfloat16 or float16, got %s" % Y.dtype)
    if table.dtype not in (torch.float32, Y.dtype):
        raise TypeError("table must be float32 or %s, got %s" % (Y.dtype, table.dtype))
    rc = h._lib.cdgrab_embed(h._h, rows, vocab, width, _ids(ids, ids.shape, dev), _ELEM[table.dtype], pt, st, scale,
                             _ELEM[Y.dtype], py, sy)
    if rc:
        h._check(rc)
    return Y


def cdgrab_pergrad_embed(h: Handle, ids: torch.Tensor, dY: torch.Tensor, vocab: int, scale: float = 1.0,
                         first: Optional[torch.Tensor] = None, count: Optional[torch.Tensor] = None,
                         tokens: Optional[int] = None, G_out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Per-example gradients G[examples][vocab * width] of cdgrab_embed's table from its output's gradients dY; rows of
    examples as in cdgrab_pergrad_layernorm, an id per row."""
    dev = h.device
    py, rows, width, sy = _rows(dY, "dY", dev)
    t = _token_rows(dY, rows, first, count, tokens, dev)
    G, sg = _grad_rows(h, G_out, t.examples, vocab * width)
    rc = h._lib.cdgrab_pergrad_embed(h._h, ctypes.byref(t), vocab, width, _ELEM[dY.dtype], _ids(ids, dY.shape[:-1], dev), py, sy,
                                     scale, G.data_ptr(), sg)
    if rc:
        h._check(rc)
    return G


def _heads(width: int, q_heads: int, k_heads: int, base: float, eps: float) -> _Heads:
    heads = q_heads + k_heads
    if q_heads < 0 or k_heads < 0 or heads < 1 or width % heads:
        raise ValueError("rows of %d features are not those of %d + %d heads" % (width, q_heads, k_heads))
    return _Heads(q_heads, k_heads, width // heads, base, eps)


def cdgrab_headnorm(h: Handle, X: torch.Tensor, gain_q: Optional[torch.Tensor] = None,
                    gain_k: Optional[torch.Tensor] = None, *, q_heads: int, k_heads: int, eps: float = 1e-6,
                    base: float = 10000.0, first: Optional[torch.Tensor] = None, count: Optional[torch.Tensor] = None,
                    tokens: Optional[int] = None, Y: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Norm of every head's features (root mean square, gains [dim] float32 for queries and keys) and rotation by the row's
    position in its example (``base`` 0: none).  X[..., (q_heads + k_heads) * dim] holds the queries' heads and behind them the
    keys'; rows of examples as in cdgrab_pergrad_layernorm.  Rows of no example keep what Y holds (zero where the call makes Y)."""
    dev = h.device
    px, rows, width, sx = _rows(X, "X", dev)
    t = _token_rows(X, rows, first, count, tokens, dev)
    s = _heads(width, q_heads, k_heads, base, eps)
    if Y is None:
        Y = _made_like(h, X, X.shape, X.dtype, first is not None or count is not None)
        py, sy = Y.data_ptr(), width or 1
    else:
        py, _, _, sy = _rows(Y, "Y", dev, X)
    rc = h._lib.cdgrab_headnorm(h._h, ctypes.byref(t), ctypes.byref(s), _ELEM[X.dtype], px, sx,
                                _vector(gain_q, s.dim, "gain_q", dev), _vector(gain_k, s.dim, "gain_k", dev), py, sy)
    if rc:
        h._check(rc)
    return Y


def cdgrab_pergrad_headnorm(h: Handle, X: torch.Tensor, dY: torch.Tensor, gain_q: Optional[torch.Tensor] = None,
                            gain_k: Optional[torch.Tensor] = None, *, q_heads: int, k_heads: int, eps: float = 1e-6,
                            base: float = 10000.0, first: Optional[torch.Tensor] = None,
                            count: Optional[torch.Tensor] = None, tokens: Optional[int] = None,
                            dX: Optional[torch.Tensor] = None, G_out: Optional[torch.Tensor] = None,
                            want_dx: bool = True, want_grads: bool = True):
    """Backward pass of cdgrab_headnorm: (dX, G), G[examples][gain_q's gradient | gain_k's gradient], 2 * dim wide."""
    dev = h.device
    px, rows, width, sx = _rows(X, "X", dev)
    py, _, _, sy = _rows(dY, "dY", dev, X)
    t = _token_rows(X, rows, first, count, tokens, dev)
    s = _heads(width, q_heads, k_heads, base, eps)
    pd, sd = None, width
    if dX is not None:
        pd, _, _, sd = _rows(dX, "dX", dev, X)
    elif want_dx:
        dX = _made_like(h, X, X.shape, X.dtype, first is not None or count is not None)
        pd, sd = dX.data_ptr(), width or 1
    G, pg, sg = None, None, 0
    if G_out is not None or want_grads:
        G, sg = _grad_rows(h, G_out, t.examples, 2 * s.dim)
        pg = G.data_ptr()
    rc = h._lib.cdgrab_pergrad_headnorm(h._h, ctypes.byref(t), ctypes.byref(s), _ELEM[X.dtype], px, sx, py, sy,
                                        _vector(gain_q, s.dim, "gain_q", dev), _vector(gain_k, s.dim, "gain_k", dev), pd, sd,
                                        pg, sg)
    if rc:
        h._check(rc)
    return dX, G


def _attention_rows(h, Q, K, V, q_heads, kv_heads, scale, first, count, tokens):
    """(spans, head dim, scale, pointer and stride of Q, K and V, leading shape)"""
    dev = h.device
    pq, rows, qw, sq = _rows(Q, "Q", dev)
    if q_heads < 1 or kv_heads < 1 or q_heads % kv_heads or qw % q_heads:
        raise ValueError("rows of %d features and %d heads of queries on %d of keys do not go together" % (qw, q_heads, kv_heads))
    dim, lead, kind = qw // q_heads, Q.shape[:-1], Q.dtype
    kw = kv_heads * dim
    pk, _, wk, sk = _rows(K, "K", dev)
    pv, _, wv, sv = _rows(V, "V", dev)
    for x, w, name in ((K, wk, "K"), (V, wv, "V")):
        if x.dtype is not kind or w != kw or x.shape[:-1] != lead:
            raise ValueError("%s must be %s %s, got %s %s" % (name, kind, (*lead, kw), x.dtype, tuple(x.shape)))
    if scale is None:
        scale = dim ** -0.5 if dim else 1.0
    return _token_rows(Q, rows, first, count, tokens, dev), dim, scale, (pq, sq, pk, sk, pv, sv), lead


def _rows_or_made(h, t, name, like, partly):
    """(tensor, pointer, stride) of an output of the type and shape of `like`."""
    if t is None:
        t = _made_like(h, like, like.shape, like.dtype, partly)
        return t, t.data_ptr(), like.shape[-1] or 1
    p, _, _, s = _rows(t, name, h.device, like)
    return t, p, s


def cdgrab_attention(h: Handle, Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, *, q_heads: int, kv_heads: int,
                     scale: Optional[float] = None, first: Optional[torch.Tensor] = None,
                     count: Optional[torch.Tensor] = None, tokens: Optional[int] = None, O: Optional[torch.Tensor] = None,
                     want_lse: bool = True):
    """Causal attention within each example: (O, lse).  Q[..., q_heads * dim], K and V[..., kv_heads * dim], lse[q_heads, ...]
    float32 (logarithms of the sums, for the backward pass); ``scale`` is 1 / sqrt(dim) by default; rows of examples as in
    cdgrab_pergrad_layernorm.  Rows of no example keep what O holds (zero where the call makes it, and in lse)."""
    t, dim, scale, at, lead = _attention_rows(h, Q, K, V, q_heads, kv_heads, scale, first, count, tokens)
    partly = first is not None or count is not None
    O, po, so = _rows_or_made(h, O, "O", Q, partly)
    lse = _made_like(h, Q, (q_heads, *lead), torch.float32, partly) if want_lse else None
    rc = h._lib.cdgrab_attention(h._h, ctypes.byref(t), q_heads, kv_heads, dim, _ELEM[Q.dtype], scale, *at, po, so,
                                 lse.data_ptr() if want_lse else None)
    if rc:
        h._check(rc)
    return O, lse


def cdgrab_attention_backward(h: Handle, Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, O: torch.Tensor,
                              lse: torch.Tensor, dO: torch.Tensor, *, q_heads: int, kv_heads: int,
                              scale: Optional[float] = None, first: Optional[torch.Tensor] = None,
                              count: Optional[torch.Tensor] = None, tokens: Optional[int] = None,
                              dQ: Optional[torch.Tensor] = None, dK: Optional[torch.Tensor] = None,
                              dV: Optional[torch.Tensor] = None):
    """Backward pass of cdgrab_attention from its outputs O and lse and the gradient dO: (dQ, dK, dV), which may be given, as
    stretches of one array's rows too.  Rows of no example keep what they hold (zero where the call makes them).  Gradients are
    good where scores (scale * Q . K) are at most 65 536 in size."""
    t, dim, scale, at, lead = _attention_rows(h, Q, K, V, q_heads, kv_heads, scale, first, count, tokens)
    po, _, _, so = _rows(O, "O", h.device, Q)
    pg, _, _, sg = _rows(dO, "dO", h.device, Q)
    pl = _ptr(lse, torch.float32, (q_heads, *lead), "lse", h.device)
    partly = first is not None or count is not None
    dQ, pq, sq = _rows_or_made(h, dQ, "dQ", Q, partly)
    dK, pk, sk = _rows_or_made(h, dK, "dK", K, partly)
    dV, pv, sv = _rows_or_made(h, dV, "dV", V, partly)
    rc = h._lib.cdgrab_attention_backward(h._h, ctypes.byref(t), q_heads, kv_heads, dim, _ELEM[Q.dtype], scale, *at, po, so, pl,
                                          pg, sg, pq, sq, pk, sk, pv, sv)
    if rc:
        h._check(rc)
    return dQ, dK, dV


def cdgrab_train_epoch_softmax_orthogonal(h: Handle, X: torch.Tensor, y: torch.Tensor, W: torch.Tensor,
                                          velocity: torch.Tensor, perm_in: Optional[torch.Tensor] = None,
                                          lr: float = 0.02, momentum: float = 0.95, steps: int = 5, coeffs=None,
                                          want_grads: bool = False, want_loss: bool = True) -> dict:
    """cdgrab_train_epoch_softmax with W <- W - lr O(velocity), O as cdgrab_orthogonalize makes it of the
    velocity [(in_dim+1)*classes] as a matrix of the shape of W."""
    m, n, in_dim = X.shape
    classes = W.shape[1]
    d = (in_dim + 1) * classes
    dev = h.device
    empty = _allocator(h)
    signs = empty((m, n // 2), dtype=torch.int8, device=dev)
    perm = empty((m, n), dtype=torch.int32, device=dev)
    grads = empty((m, n, d), dtype=torch.float32, device=dev) if want_grads else None
    loss = empty((m, n), dtype=torch.float32, device=dev) if want_loss else None
    h._check(h._lib.cdgrab_train_epoch_softmax_orthogonal(
        h._h, m, n, in_dim, classes,
        _ptr(X, torch.float32, (m, n, in_dim), "X", dev), _ptr(y, torch.int32, (m, n), "y", dev),
        _ptr(perm_in, torch.int32, (m, n), "perm_in", dev),
        _ptr(W, torch.float32, (in_dim + 1, classes), "W", dev),
        _ptr(velocity, torch.float32, (d,), "velocity", dev), lr, momentum, steps, _coeffs(coeffs),
        signs.data_ptr(), perm.data_ptr(),
        grads.data_ptr() if grads is not None else None,
        loss.data_ptr() if loss is not None else None))
    return {"signs": signs, "perm": perm, "grads": grads, "loss": loss}
