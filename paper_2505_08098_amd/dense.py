"""Dense attention beside the sparse operator: cross attention over a ragged
batch, and attention over an 8-bit key/value cache (include/f3s_cross.h,
include/f3s_cache.h).  Argument marshalling only, like ``binding``: results carry
no autograd graph, also where an operand requires gradients.

    plan = f3s.CrossPlan(q_ptr, k_ptr, heads, kv_heads, d)     # once per batch
    O, lse = f3s.cross_forward(plan, Q, K, V)
    dQ, dK, dV = f3s.cross_backward(plan, Q, K, V, O, dO, lse)

    cache = f3s.Cache.empty(n_pages, page_size, kv_heads, d)
    f3s.cache_write(cache, K, V, table, lens)                  # the newest tokens
    O, lse = f3s.cache_attend(cache, Q, table, lens, prefix=pages, prefix_len=n)
"""
import contextlib
import ctypes
import functools
import math

import torch

from .binding import (_DTYPE_CODE, _TENSORS, F3SError, _BuildOn, _check_device_tensor,
                      _empty_like, _raw_stream, load_library)

_LIB = None
_vp, _i32, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
_HALF = (torch.float16, torch.bfloat16)
_READ_TYPES = _HALF + (torch.float32,)
_MOST = 2**31 - 1


class _CacheStruct(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("k_exp", _vp), ("v_exp", _vp), ("n_pages", _i32),
                ("n_kv_heads", _i32), ("page_size", _i32), ("d", _i32)]


def _lib():
    global _LIB
    if _LIB is None:
        L = load_library()
        cache = ctypes.POINTER(_CacheStruct)
        for name, res, args in (
                ("f3s_cross_plan", _vp, [_vp, _vp, _vp, _vp, _i32, _i32, _i32, _i32]),
                ("f3s_cross_destroy", None, [_vp]),
                ("f3s_cross_forward_workspace_bytes", _sz, [_vp]),
                ("f3s_cross_backward_workspace_bytes", _sz, [_vp]),
                ("f3s_cross_forward", ctypes.c_int,
                 [_vp] * 4 + [_i32, _vp, _vp, ctypes.c_float, _vp, _sz, _vp]),
                ("f3s_cross_backward", ctypes.c_int,
                 [_vp] * 4 + [_i32] + [_vp] * 6 + [ctypes.c_float, _vp, _sz, _vp]),
                ("f3s_cache_write", ctypes.c_int,
                 [cache, _vp, _vp, _i32, _vp, _i32, _vp, _i32, _i32, _vp]),
                ("f3s_cache_read", ctypes.c_int,
                 [cache, _vp, _vp, _i32, _vp, _i32, _vp, _i32, _i32, _vp]),
                ("f3s_cache_attend", ctypes.c_int,
                 [cache, _vp, _i32, _vp, _vp, _vp, _i32, _vp, _i32, _i32, _i32, _vp, _i32,
                  ctypes.c_float, _vp, _sz, _vp]),
                ("f3s_cache_attend_workspace_bytes", _sz, [cache] + [_i32] * 5)):
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _LIB = L
    return _LIB


@contextlib.contextmanager
def _switch(device, stream):
    with torch.cuda.device(device):
        with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
            yield


# The current device (torch's own accessor where it has one: 0.1 us instead of 0.5).
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _elsewhere(device, stream):
    """None where a call runs as it is; else what makes its device and stream
    current, so that results and workspaces are the stream's own memory (torch
    hands a stream's freed memory to that stream's later work only)."""
    if stream is None:
        return None if _current_device() == device.index else _switch(device, None)
    if stream.device != device:
        raise ValueError(f"the stream is on {stream.device}, the operands on {device}")
    return _switch(device, stream)


def _on_its_device(fn):
    """The call with its device and stream current; fn takes a plan or a cache
    first and no stream."""
    @functools.wraps(fn)
    def call(handle, *args, stream=None, **kwargs):
        switch = _elsewhere(handle.device, stream)
        if switch is None:
            return fn(handle, *args, **kwargs)
        with switch:
            return fn(handle, *args, **kwargs)
    return call


def _check(t, name, dtype, device, shape):
    if (type(t) in _TENSORS and t.dtype is dtype and t.shape == shape and t.device == device
            and t.is_contiguous()):
        return
    _check_device_tensor(t, name, dtype, device)
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")


def _dtype_of(t, name):
    if not isinstance(t, torch.Tensor) or t.dtype not in _HALF:
        raise TypeError(f"{name} must be a float16 or bfloat16 device tensor")
    return t.dtype


def _fail(rc, name):
    raise F3SError(rc, name)


def _host_ints(x, name):
    import numpy as np
    a = np.asarray(x)
    if a.ndim != 1 or (a.size and a.dtype.kind not in "iu"):
        raise ValueError(f"{name} must be a host sequence of whole numbers")
    if a.size and (a.min() < 0 or a.max() > _MOST):
        raise ValueError(f"{name} must lie in [0, 2^31)")
    return np.ascontiguousarray(a, dtype=np.int32)


def _size(x, name):
    """x as an int that 32 bits hold (ctypes would take it modulo 2^32)."""
    x = int(x)
    if not -_MOST <= x <= _MOST:
        raise ValueError(f"{name} must be a 32-bit number, got {x}")
    return x


# ---- cross attention ----------------------------------------------------------

class CrossPlan:
    """f3s_cross_plan: the work of a ragged batch.  Sequence b has the rows
    q_ptr[b] .. q_ptr[b+1] - 1 of Q and k_ptr[b] .. k_ptr[b+1] - 1 of K and V
    (host sequences of ints, first 0); with q_len / k_len only the first of
    them, the others being padding.  ``heads`` query heads share ``kv_heads``
    key heads (default: as many), ``d`` values each."""

    def __init__(self, q_ptr, k_ptr, heads, kv_heads=None, d=64, q_len=None, k_len=None,
                 device="cuda"):
        self._h = None
        L = _lib()
        q, k = _host_ints(q_ptr, "q_ptr"), _host_ints(k_ptr, "k_ptr")
        if q.size < 1 or k.size != q.size:
            raise ValueError("q_ptr and k_ptr must hold one entry more than sequences")
        lens = [None if x is None else _host_ints(x, n)
                for x, n in ((q_len, "q_len"), (k_len, "k_len"))]
        if any(x is not None and x.size != q.size - 1 for x in lens):
            raise ValueError("q_len and k_len must hold one entry per sequence")
        heads, d = _size(heads, "heads"), _size(d, "d")
        kv_heads = heads if kv_heads is None else _size(kv_heads, "kv_heads")
        device = torch.device(device)
        if device.type != "cuda":
            raise ValueError("the plan's device must be a GPU")
        if device.index is None:
            device = torch.device("cuda", torch.cuda.current_device())
        ptr = lambda a: None if a is None else a.ctypes.data_as(_vp)
        with _BuildOn(device):
            h = L.f3s_cross_plan(ptr(q), ptr(k), ptr(lens[0]), ptr(lens[1]), q.size - 1,
                                 heads, kv_heads, d)
        if not h:
            raise F3SError(L.f3s_last_error(), "f3s_cross_plan")
        self._h = h
        self.device = device
        self.heads, self.kv_heads, self.d = heads, kv_heads, d
        self.q_shape = (int(q[-1]), self.heads, self.d)
        self.k_shape = (int(k[-1]), self.kv_heads, self.d)
        self.lse_shape = self.q_shape[:2]
        self.scale = 1.0 / math.sqrt(self.d)
        self._forward_bytes = L.f3s_cross_forward_workspace_bytes(h)
        self._backward_bytes = L.f3s_cross_backward_workspace_bytes(h)

    @property
    def handle(self):
        if self._h is None:
            raise RuntimeError("plan was destroyed")
        return self._h

    def close(self):
        if self._h is not None:
            _lib().f3s_cross_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


def _cross_operands(plan, Q, K, V):
    dtype = _dtype_of(Q, "Q")
    _check(Q, "Q", dtype, plan.device, plan.q_shape)
    _check(K, "K", dtype, plan.device, plan.k_shape)
    _check(V, "V", dtype, plan.device, plan.k_shape)
    return dtype


@_on_its_device
def cross_forward(plan, Q, K, V, scale=None, out=None, lse=None):
    """f3s_cross_forward: O = softmax(scale Q K^T) V within each sequence of
    the plan.  Q [rows, heads, d], K and V [rows, kv_heads, d], fp16 or bf16;
    ``stream=`` (default: torch's current one).  Returns (O, lse): O like Q,
    lse fp32 [rows, heads]."""
    dtype = _cross_operands(plan, Q, K, V)
    device = plan.device
    if out is None:
        out = _empty_like(Q, dtype)
    else:
        _check(out, "out", dtype, device, plan.q_shape)
    if lse is None:
        lse = torch.empty(plan.lse_shape, dtype=torch.float32, device=device)
    else:
        _check(lse, "lse", torch.float32, device, plan.lse_shape)
    nbytes = plan._forward_bytes
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None
    rc = _lib().f3s_cross_forward(
        plan.handle, Q.data_ptr(), K.data_ptr(), V.data_ptr(), _DTYPE_CODE[dtype],
        out.data_ptr(), lse.data_ptr(), plan.scale if scale is None else float(scale),
        ws.data_ptr() if nbytes else None, nbytes, _raw_stream(device.index))
    if rc:
        _fail(rc, "f3s_cross_forward")
    return out, lse


@_on_its_device
def cross_backward(plan, Q, K, V, O, dO, lse, scale=None):
    """f3s_cross_backward: (dQ, dK, dV), of the operands' shapes and type, for
    dO = dL/dO and the forward's O and lse; ``stream=`` as cross_forward."""
    dtype = _cross_operands(plan, Q, K, V)
    device = plan.device
    _check(O, "O", dtype, device, plan.q_shape)
    _check(dO, "dO", dtype, device, plan.q_shape)
    _check(lse, "lse", torch.float32, device, plan.lse_shape)
    dQ, dK, dV = _empty_like(Q, dtype), _empty_like(K, dtype), _empty_like(V, dtype)
    nbytes = plan._backward_bytes
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None
    rc = _lib().f3s_cross_backward(
        plan.handle, Q.data_ptr(), K.data_ptr(), V.data_ptr(), _DTYPE_CODE[dtype],
        O.data_ptr(), dO.data_ptr(), lse.data_ptr(), dQ.data_ptr(), dK.data_ptr(),
        dV.data_ptr(), plan.scale if scale is None else float(scale),
        ws.data_ptr() if nbytes else None, nbytes, _raw_stream(device.index))
    if rc:
        _fail(rc, "f3s_cross_backward")
    return dQ, dK, dV


# ---- the cache -------------------------------------------------------------------

class Cache:
    """Pages of keys and values in 8 bits: codes ``k`` and ``v``
    (float8_e4m3fn, [pages, kv_heads, page_size, d]) and a power of two for
    each row, ``k_exp`` and ``v_exp`` (uint8, [pages, kv_heads, page_size]:
    value = code * 2^(exp - 127)).  The tensors are the caller's and stay where
    they are: another place for them is another Cache."""

    def __init__(self, k, v, k_exp, v_exp):
        if not isinstance(k, torch.Tensor) or k.dim() != 4:
            raise ValueError("k must be a [pages, kv_heads, page_size, d] device tensor")
        for t, n in ((k, "k"), (v, "v")):
            _check_device_tensor(t, n, torch.float8_e4m3fn, k.device)
        for t, n in ((k_exp, "k_exp"), (v_exp, "v_exp")):
            _check_device_tensor(t, n, torch.uint8, k.device)
        if v.shape != k.shape or k_exp.shape != k.shape[:3] or v_exp.shape != k.shape[:3]:
            raise ValueError("k and v must share one shape, k_exp and v_exp its first three")
        self._tensors = (k, v, k_exp, v_exp)
        self.device = k.device
        self.n_pages, self.kv_heads, self.page_size, self.d = k.shape
        if max(k.shape) > _MOST:
            raise ValueError("more than 2^31 - 1 pages, heads, tokens or values")
        self._struct = _CacheStruct(k.data_ptr(), v.data_ptr(), k_exp.data_ptr(),
                                    v_exp.data_ptr(), self.n_pages, self.kv_heads,
                                    self.page_size, self.d)
        self._ref = ctypes.byref(self._struct)
        self.scale = 1.0 / math.sqrt(self.d) if self.d else 1.0
        self._bytes = {}  # workspace of an attend call, by its sizes

    # (read-only: the struct holds their addresses)
    k = property(lambda self: self._tensors[0])
    v = property(lambda self: self._tensors[1])
    k_exp = property(lambda self: self._tensors[2])
    v_exp = property(lambda self: self._tensors[3])

    @classmethod
    def empty(cls, n_pages, page_size, kv_heads, d, device="cuda"):
        """A cache of new pages, all zeros."""
        shape = (int(n_pages), int(kv_heads), int(page_size), int(d))
        codes = [torch.zeros(shape, dtype=torch.uint8, device=device)
                 .view(torch.float8_e4m3fn) for _ in range(2)]
        powers = [torch.zeros(shape[:3], dtype=torch.uint8, device=device) for _ in range(2)]
        return cls(*codes, *powers)


def _sequences(cache, table, lens):
    """(number of sequences, pages of a table row), checked."""
    device = cache.device
    for t, n in ((table, "table"), (lens, "lens")):
        if not (type(t) in _TENSORS and t.dtype is torch.int32 and t.device == device
                and t.is_contiguous()):
            _check_device_tensor(t, n, torch.int32, device)
    if table.dim() != 2 or lens.dim() != 1 or table.shape[0] != lens.shape[0]:
        raise ValueError("table must be [sequences, pages], lens [sequences]")
    if table.shape[1] > _MOST or table.shape[0] > _MOST:
        raise ValueError("more than 2^31 - 1 sequences, or pages of one")
    return table.shape


@_on_its_device
def cache_write(cache, K, V, table, lens):
    """f3s_cache_write: the newest rows of every sequence, K and V [sequences,
    n, kv_heads, d] in fp16 or bf16, quantised into the pages of ``table``
    (int32 [sequences, pages]).  ``lens`` (int32) are the sequences' lengths
    with these rows; row t goes to position lens[b] - n + t.  ``stream=``
    (default: torch's current one)."""
    B, pages = _sequences(cache, table, lens)
    dtype = _dtype_of(K, "K")
    if K.dim() != 4:
        raise ValueError("K must be [sequences, n, kv_heads, d]")
    n = _size(K.shape[1], "n")
    shape = (B, n, cache.kv_heads, cache.d)
    _check(K, "K", dtype, cache.device, shape)
    _check(V, "V", dtype, cache.device, shape)
    rc = _lib().f3s_cache_write(
        cache._ref, K.data_ptr(), V.data_ptr(), _DTYPE_CODE[dtype], table.data_ptr(), pages,
        lens.data_ptr(), B, n, _raw_stream(cache.device.index))
    if rc:
        _fail(rc, "f3s_cache_write")


@_on_its_device
def cache_read(cache, table, lens, n, dtype=torch.float16):
    """f3s_cache_read: the ``n`` newest rows of every sequence, (K, V) of
    ``dtype`` (float16, bfloat16 or float32), [sequences, n, kv_heads, d];
    ``stream=`` as cache_write."""
    B, pages = _sequences(cache, table, lens)
    if dtype not in _READ_TYPES:
        raise TypeError("dtype must be float16, bfloat16 or float32")
    n = _size(n, "n")
    shape = (B, n, cache.kv_heads, cache.d)
    K = torch.empty(shape, dtype=dtype, device=cache.device)
    V = torch.empty_like(K)
    rc = _lib().f3s_cache_read(
        cache._ref, K.data_ptr(), V.data_ptr(), _DTYPE_CODE[dtype], table.data_ptr(), pages,
        lens.data_ptr(), B, n, _raw_stream(cache.device.index))
    if rc:
        _fail(rc, "f3s_cache_read")
    return K, V


@_on_its_device
def cache_attend(cache, Q, table, lens, prefix=None, prefix_len=0, scale=None, out=None,
                 lse=None):
    """f3s_cache_attend: the newest tokens of every sequence, Q [sequences, n,
    heads, d] in fp16 or bf16, attend to the first ``prefix_len`` tokens of the
    pages ``prefix`` (int32, shared by all sequences) and to their own cached
    keys up to themselves; ``stream=`` as cache_write.  Returns (O, lse): O
    like Q, lse fp32 [sequences, n, heads]."""
    B, pages = _sequences(cache, table, lens)
    dtype = _dtype_of(Q, "Q")
    if Q.dim() != 4 or Q.shape[2] < 1 or Q.shape[2] % cache.kv_heads:
        raise ValueError("Q must be [sequences, n, heads, d], heads a multiple of kv_heads")
    _, n, heads, _ = shape = Q.shape
    device = cache.device
    _check(Q, "Q", dtype, device, (B, n, heads, cache.d))
    if prefix is None:
        if prefix_len != 0:
            raise ValueError("prefix and a positive prefix_len come together")
    else:
        prefix_len = _size(prefix_len, "prefix_len")
        _check_device_tensor(prefix, "prefix", torch.int32, device)
        if prefix_len < 1:
            raise ValueError("prefix and a positive prefix_len come together")
        if prefix.dim() != 1 or prefix.numel() * cache.page_size < prefix_len:
            raise ValueError("prefix must name enough pages for prefix_len tokens")
    sizes = (pages, B, n, heads, prefix_len)
    nbytes = cache._bytes.get(sizes)
    if nbytes is None:
        if max(sizes) > _MOST:
            raise ValueError("more than 2^31 - 1 tokens or heads")
        if len(cache._bytes) >= 64:  # (a prefix that grows)
            cache._bytes.clear()
        nbytes = _lib().f3s_cache_attend_workspace_bytes(cache._ref, *sizes)
        cache._bytes[sizes] = nbytes
    if out is None:
        out = _empty_like(Q, dtype)
    else:
        _check(out, "out", dtype, device, shape)
    if lse is None:
        lse = torch.empty((B, n, heads), dtype=torch.float32, device=device)
    else:
        _check(lse, "lse", torch.float32, device, (B, n, heads))
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None
    rc = _lib().f3s_cache_attend(
        cache._ref, Q.data_ptr(), _DTYPE_CODE[dtype], out.data_ptr(), lse.data_ptr(),
        table.data_ptr(), pages, lens.data_ptr(), B, n, heads,
        None if prefix is None else prefix.data_ptr(), prefix_len,
        cache.scale if scale is None else float(scale), ws.data_ptr() if nbytes else None,
        nbytes, _raw_stream(device.index))
    if rc:
        _fail(rc, "f3s_cache_attend")
    return out, lse
