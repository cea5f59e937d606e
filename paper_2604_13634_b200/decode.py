"""ctypes binding of the decode-pass operators: rotary positions, the paged cache, attention over it.

Like binding.py: argument marshalling only, one function per entry point of include/csd.h, every failure raises.
"""

from __future__ import annotations

from ctypes import POINTER, Structure, byref, c_double, c_float, c_int, c_int64, c_size_t, c_uint64, c_void_p

import torch

from .binding import CSD_BF16, CSD_F16, CSD_F32, CsdError, _check, _ptr, lib

CACHE_FULL, CACHE_ROW_FULL, CACHE_BAD_PAGE, CACHE_BAD_ROW, CACHE_INTERNAL = 1, 2, 4, 8, 16

_DTYPES = {torch.float32: CSD_F32, torch.bfloat16: CSD_BF16, torch.float16: CSD_F16}
_LAYOUTS = {"half": 0, "interleaved": 1}
_SCALINGS = {"none": 0, "linear": 1, "base": 2, "parts": 3, "yarn": 4}
_RANGES = {"parts": (1.0, 4.0), "yarn": (1.0, 32.0)}          # turns: pairs that make fewer are stretched, more are kept


class RopeStruct(Structure):
    _fields_ = [("steps", c_void_p), ("rot", c_int), ("layout", c_int), ("magnitude", c_float)]


class CacheStruct(Structure):
    _fields_ = [("k", c_void_p), ("v", c_void_p), ("dtype", c_int), ("layers", c_int), ("n_pages", c_int), ("page_size", c_int),
                ("heads", c_int), ("dim", c_int), ("stride_layer", c_int64), ("stride_page", c_int64), ("stride_head", c_int64),
                ("stride_token", c_int64), ("rows", c_int), ("max_pages", c_int), ("meta", c_void_p), ("scratch", c_void_p)]


class CacheLayout(Structure):
    _fields_ = [(n, c_size_t) for n in ("flags", "lens", "granted", "table", "refs", "free_bits", "total")]


_strides3 = [c_int64] * 3
SIGNATURES = {
    "csd_rope_steps": (c_int, [c_int, c_double, c_int, c_double, c_double, c_double, c_double, POINTER(c_uint64), POINTER(c_float)]),
    "csd_rope": (c_int, [c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_int, *_strides3, *_strides3, c_void_p, c_int64, c_int64,
                         POINTER(RopeStruct), c_int, c_void_p]),
    "csd_rope_append": (c_int, [c_void_p, *_strides3, c_int, c_void_p, *_strides3, c_void_p, *_strides3, c_void_p, c_int,
                                POINTER(CacheStruct), c_int, POINTER(RopeStruct), c_void_p, c_void_p]),
    "csd_cache_meta_bytes": (c_size_t, [c_int, c_int, c_int]),
    "csd_cache_meta_layout": (c_int, [c_int, c_int, c_int, POINTER(CacheLayout)]),
    "csd_cache_scratch_bytes": (c_size_t, [c_int, c_int, c_int]),
    "csd_cache_rebuild": (c_int, [POINTER(CacheStruct), c_void_p]),
    "csd_cache_extend": (c_int, [POINTER(CacheStruct), c_int, c_void_p, c_void_p]),
    "csd_cache_truncate": (c_int, [POINTER(CacheStruct), c_void_p, c_void_p]),
    "csd_cache_commit": (c_int, [POINTER(CacheStruct), c_void_p, c_void_p]),
    "csd_cache_fork": (c_int, [POINTER(CacheStruct), c_void_p, c_void_p]),
    "csd_cache_compact": (c_int, [POINTER(CacheStruct), c_void_p]),
    "csd_attention_workspace_bytes": (c_size_t, [c_int] * 5),
    "csd_attention": (c_int, [c_void_p, *_strides3, c_int, c_int, POINTER(CacheStruct), c_int, c_float, c_void_p, c_void_p, c_void_p,
                              c_void_p, c_size_t, c_void_p]),
}

_current_device = torch._C._cuda_getDevice


def _stream_ptr(stream, device: int) -> int:
    """The stream asked for, or the device's current one (the raw handle: a Stream object costs 3 us to make, as much as the
    call that it is made for).  The device of the call's tensors has to be the current one: a kernel given another device's addresses
    would fault."""
    if device != _current_device():
        raise CsdError(f"tensors on device {device}, but the current device is {_current_device()}")
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device)
    if stream.device_index != device:
        raise CsdError(f"tensors on device {device}, but a stream of device {stream.device_index}")
    return stream.cuda_stream


def _scattered(what: str, *devices: int):
    raise CsdError(f"{what}: tensors on different devices: {devices} (-1: the host)")


def _result(x, stream, **kw):
    """An uninitialised result like x, owned by the stream that writes it: memory of the current stream could have been freed by
    work that is still to run there, and would go back to it while the other stream still writes."""
    if stream is None:
        return torch.empty_like(x, **kw)
    with torch.cuda.stream(stream):
        return torch.empty_like(x, **kw)


_typed = None


def _lib():
    global _typed
    if _typed is None:
        L = lib()
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _typed = L
    return _typed


def csd_rope_steps(rot: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, original_len: float = 8192,
                   low: float | None = None, high: float | None = None):
    """(steps, magnitude): the rotation per position of each pair as a 64-bit fraction of a turn (an int64 CPU tensor
    with the same bits), and the factor on turned elements."""
    if scaling not in _SCALINGS:
        raise CsdError(f"unknown scaling {scaling!r}: one of {sorted(_SCALINGS)}")
    lo, hi = _RANGES.get(scaling, (1.0, 2.0))
    steps = (c_uint64 * max(1, rot // 2))()
    magnitude = c_float()
    _check(_lib().csd_rope_steps(rot, base, _SCALINGS[scaling], factor, original_len, lo if low is None else low, hi if high is None else high,
                                 steps, byref(magnitude)), "csd_rope_steps")
    return torch.frombuffer(steps, dtype=torch.int64).clone(), float(magnitude.value)


class RopePlan:
    """A rotation in device memory: `rot` elements of every head, frequencies base^(-2i/rot), scaled for long contexts."""

    def __init__(self, rot: int, base: float = 10000.0, layout: str = "half", scaling: str = "none", factor: float = 1.0,
                 original_len: float = 8192, low: float | None = None, high: float | None = None, device="cuda"):
        if layout not in _LAYOUTS:
            raise CsdError(f"unknown layout {layout!r}: one of {sorted(_LAYOUTS)}")
        steps, self.magnitude = csd_rope_steps(rot, base, scaling, factor, original_len, low, high)
        self.rot, self.layout = rot, layout
        self.steps = steps.to(device)
        self._device = self.steps.get_device()
        self._struct = RopeStruct(self.steps.data_ptr(), rot, _LAYOUTS[layout], self.magnitude)
        self._ref = byref(self._struct)


class _Rope(torch.autograd.Function):
    """The rotation is linear: its gradient is the turn back, with the same factor."""

    @staticmethod
    def forward(ctx, x, positions, plan, inverse, stream):
        ctx.save_for_backward(positions)
        ctx.plan, ctx.inverse = plan, inverse
        return csd_rope(x, positions, plan, inverse=inverse, stream=stream)

    @staticmethod
    def backward(ctx, g):
        (positions,) = ctx.saved_tensors
        g = g if g.stride(3) == 1 else g.contiguous()
        return csd_rope(g, positions, ctx.plan, inverse=not ctx.inverse), None, None, None, None


def csd_rope(x, positions, plan: RopePlan, out=None, inverse: bool = False, stream=None):
    """x [B, S, H, D] turned by positions [B, S] int32 (or [S], shared by the batch); `inverse` turns back, which is the
    gradient: autograd knows it where x requires one and no `out` is given.  `out` may be x itself.  Returns out."""
    if x.requires_grad and torch.is_grad_enabled():
        if out is not None:
            raise CsdError("csd_rope: a result written into `out` has no gradient; x requires one")
        return _Rope.apply(x, positions, plan, inverse, stream)
    code = _DTYPES.get(x.dtype)
    if code is None:
        raise CsdError(f"x must be float32, bfloat16 or float16, got {x.dtype}")
    out = _result(x, stream) if out is None else out
    B, S, H, D = shape = x.shape
    xs, ys, ps = x.stride(), out.stride(), positions.stride()
    assert positions.dtype == torch.int32 and xs[3] == 1
    assert out.shape == shape and out.dtype == x.dtype and ys[3] == 1
    dev = plan._device
    if not (x.get_device() == out.get_device() == positions.get_device() == dev >= 0):
        _scattered("csd_rope", x.get_device(), out.get_device(), positions.get_device(), dev)
    if len(ps) == 1:
        assert positions.shape[0] == S
        ps = (0, ps[0])
    else:
        assert positions.shape == (B, S)
    rc = _lib().csd_rope(x.data_ptr(), out.data_ptr(), code, B, S, H, D, xs[0], xs[1], xs[2], ys[0], ys[1], ys[2], positions.data_ptr(),
                         ps[0], ps[1], plan._ref, 1 if inverse else 0, _stream_ptr(stream, dev))
    if rc:
        _check(rc, "csd_rope")
    return out


class PagedCache:
    """Keys and values of `rows` sequences in pages, with the bookkeeping on the device.

    k, v: [layers, n_pages, kv_heads, page_size, head_dim] views, each page dense (whatever lies outside within
    it: heads or tokens); pass your own to adopt them.  table, lens, granted, refs are views of `meta`: copying meta saves or restores the bookkeeping.
    """

    def __init__(self, rows: int, n_pages: int, page_size: int, layers: int, kv_heads: int, head_dim: int, dtype: torch.dtype,
                 max_len: int, k=None, v=None, token_major: bool = False, device="cuda"):
        if dtype not in (torch.bfloat16, torch.float16):
            raise CsdError(f"a cache holds bfloat16 or float16, got {dtype}")
        if page_size <= 0 or max_len <= 0:
            raise CsdError(f"unsupported page_size={page_size} max_len={max_len}")
        if (k is None) != (v is None):
            raise CsdError("a pool to adopt is both keys and values")
        shape = (layers, n_pages, kv_heads, page_size, head_dim)
        dev = k.device if k is not None else torch.device(device)
        if k is None:
            made = (layers, n_pages, page_size, kv_heads, head_dim) if token_major else shape
            k, v = (torch.zeros(made, dtype=dtype, device=dev) for _ in range(2))
            if token_major:
                k, v = k.transpose(2, 3), v.transpose(2, 3)
        assert tuple(k.shape) == shape == tuple(v.shape) and k.dtype == v.dtype == dtype and k.is_cuda and v.device == k.device
        assert k.stride() == v.stride() and k.stride(4) == 1
        self.rows, self.n_pages, self.page_size, self.layers = rows, n_pages, page_size, layers
        self.kv_heads, self.head_dim, self.dtype = kv_heads, head_dim, dtype
        self.max_pages = -(-max_len // page_size)
        self.k, self.v = k, v
        L = _lib()
        shape3 = (rows, self.max_pages, n_pages)
        bytes_ = int(L.csd_cache_meta_bytes(*shape3))
        if bytes_ == 0:
            raise CsdError(f"unsupported cache: rows={rows} max_pages={self.max_pages} n_pages={n_pages}")
        lay = CacheLayout()
        _check(L.csd_cache_meta_layout(*shape3, byref(lay)), "csd_cache_meta_layout")
        self.meta = torch.zeros(bytes_ // 4, dtype=torch.int32, device=dev)
        self.scratch = torch.empty(int(L.csd_cache_scratch_bytes(*shape3)), dtype=torch.uint8, device=dev)
        part = lambda off, n: self.meta[off // 4:off // 4 + n]  # noqa: E731
        self.lens, self.granted = part(lay.lens, rows), part(lay.granted, rows)
        self.table = part(lay.table, rows * self.max_pages).view(rows, self.max_pages)
        self.refs = part(lay.refs, n_pages)
        self._flags = part(lay.flags, 1)
        # strides of dimensions of size 1 mean nothing to torch; the library reads them
        st = list(k.stride())
        if kv_heads == 1:
            st[2] = page_size * head_dim
        if n_pages == 1:
            st[1] = kv_heads * page_size * head_dim
        self._struct = CacheStruct(k.data_ptr(), v.data_ptr(), _DTYPES[dtype], layers, n_pages, page_size, kv_heads, head_dim, st[0],
                                   st[1], st[2], st[3], rows, self.max_pages, self.meta.data_ptr(), self.scratch.data_ptr())
        self._ref = byref(self._struct)
        self._device = self.k.get_device()
        csd_cache_rebuild(self)

    def load(self, table: torch.Tensor, lens: torch.Tensor, stream=None):
        """Take over page tables [rows, <= max_pages] and lengths [rows] (a checkpoint, or pages filled elsewhere)."""
        assert table.dtype == lens.dtype == torch.int32 and table.shape[0] == self.rows == lens.shape[0]
        assert table.shape[1] <= self.max_pages
        with torch.cuda.stream(torch.cuda.current_stream() if stream is None else stream):
            self.table[:, :table.shape[1]].copy_(table)
            self.table[:, table.shape[1]:].fill_(-1)              # a length beyond the table given is flagged, not read from the one before
            self.lens.copy_(lens)
        csd_cache_rebuild(self, stream)

    def reset(self, stream=None):
        """Empty every row, free every page, clear the flags."""
        with torch.cuda.stream(torch.cuda.current_stream() if stream is None else stream):
            self.lens.zero_()
        csd_cache_rebuild(self, stream)

    def stats(self) -> dict:
        """flags, pages in use, pages shared, tokens.  Synchronises."""
        return dict(flags=int(self._flags.item()), pages=int((self.refs > 0).sum()), shared=int((self.refs > 1).sum()),
                    tokens=int(self.lens.sum()))


def _rows_arg(t, cache: PagedCache, what: str):
    if t is None:
        return None
    assert t.get_device() == cache._device and t.dtype == torch.int32 and t.shape == (cache.rows,) and t.is_contiguous(), what
    return t.data_ptr()


def csd_cache_rebuild(cache: PagedCache, stream=None):
    """Counts and free pages from cache.table and cache.lens; clears the flags."""
    _check(_lib().csd_cache_rebuild(cache._ref, _stream_ptr(stream, cache._device)), "csd_cache_rebuild")


def csd_cache_extend(cache: PagedCache, T: int, n_new=None, stream=None):
    """Room for T (or n_new[row]) more tokens in every row; cache.granted says how many each row got (all rows or none) and is the
    n_new of the calls that store and read them."""
    _check(_lib().csd_cache_extend(cache._ref, T, _rows_arg(n_new, cache, "n_new"), _stream_ptr(stream, cache._device)), "csd_cache_extend")


def csd_cache_truncate(cache: PagedCache, new_lens, stream=None):
    """Rows keep their first new_lens[row] tokens."""
    _check(_lib().csd_cache_truncate(cache._ref, _rows_arg(new_lens, cache, "new_lens"), _stream_ptr(stream, cache._device)), "csd_cache_truncate")


def csd_cache_commit(cache: PagedCache, accept_len, stream=None):
    """After a verification step: of the last extension's tokens, the first accept_len[row] + 1 stay."""
    _check(_lib().csd_cache_commit(cache._ref, _rows_arg(accept_len, cache, "accept_len"), _stream_ptr(stream, cache._device)), "csd_cache_commit")


def csd_cache_fork(cache: PagedCache, parent, stream=None):
    """Row b continues row parent[b]'s tokens (itself: unchanged; negative: empty), sharing its pages."""
    _check(_lib().csd_cache_fork(cache._ref, _rows_arg(parent, cache, "parent"), _stream_ptr(stream, cache._device)), "csd_cache_fork")


def csd_cache_compact(cache: PagedCache, stream=None):
    """The pages in use become the lowest ones."""
    _check(_lib().csd_cache_compact(cache._ref, _stream_ptr(stream, cache._device)), "csd_cache_compact")


def csd_rope_append(q, k, v, cache: PagedCache, layer: int, plan: RopePlan | None, q_out=None, n_new=None, stream=None):
    """The new tokens of a layer: q [rows, T, q_heads, D] turned into q_out (dense; returned), k turned and v as it is into
    their page slots.  plan None: no rotation.  After csd_cache_extend pass n_new=cache.granted: where that found no room it
    granted nothing, and T tokens (n_new None) would go over the newest ones of the row.  Serving form: no gradient (csd_rope has one)."""
    B, T, Hq, D = shape = q.shape
    if q_out is None:
        q_out = _result(q, stream, memory_format=torch.contiguous_format)
    qs, ks, vs = q.stride(), k.stride(), v.stride()
    assert q.dtype == k.dtype == v.dtype == q_out.dtype == cache.dtype
    assert B == cache.rows and D == cache.head_dim and k.shape == v.shape == (B, T, cache.kv_heads, D)
    assert qs[3] == ks[3] == vs[3] == 1 and q_out.shape == shape and q_out.is_contiguous()
    dev = cache._device
    if not (q.get_device() == k.get_device() == v.get_device() == q_out.get_device() == dev) or plan is not None and plan._device != dev:
        _scattered("csd_rope_append", q.get_device(), k.get_device(), v.get_device(), q_out.get_device(), dev, plan._device if plan else dev)
    rc = _lib().csd_rope_append(q.data_ptr(), qs[0], qs[1], qs[2], Hq, k.data_ptr(), ks[0], ks[1], ks[2], v.data_ptr(), vs[0], vs[1], vs[2],
                                q_out.data_ptr(), T, cache._ref, layer, None if plan is None else plan._ref,
                                None if n_new is None else _rows_arg(n_new, cache, "n_new"), _stream_ptr(stream, dev))
    if rc:
        _check(rc, "csd_rope_append")
    return q_out


class AttentionBuffers:
    """Caller-owned outputs and workspace of csd_attention for one cache, T new tokens per row and q_heads query heads."""

    def __init__(self, cache: PagedCache, T: int, q_heads: int):
        self.T, self.q_heads = T, q_heads
        dev = cache.k.device
        self.ws_bytes = int(_lib().csd_attention_workspace_bytes(cache.rows, T, q_heads, cache.kv_heads, cache.head_dim))
        if self.ws_bytes == 0:
            raise CsdError(f"unsupported attention: rows={cache.rows} T={T} q_heads={q_heads} kv_heads={cache.kv_heads} dim={cache.head_dim}")
        self.out = torch.empty(cache.rows, T, q_heads, cache.head_dim, dtype=cache.dtype, device=dev)
        self.lse = torch.empty(cache.rows, T, q_heads, dtype=torch.float32, device=dev)
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=dev)
        self._device = self.workspace.get_device()


def csd_attention(q, cache: PagedCache, layer: int, buf: AttentionBuffers, scale: float | None = None, n_new=None, stream=None):
    """buf.out, buf.lse: attention of T new tokens of every row, q [rows, T, q_heads, D], over its cache (n_new[row] > T: the first T
    of that many).  Serving form: no gradient."""
    qs = q.stride()
    assert q.dtype == cache.dtype == buf.out.dtype and qs[3] == 1 and q.shape == buf.out.shape
    assert q.shape[0] == cache.rows and q.shape[3] == cache.head_dim
    dev = cache._device
    if not (q.get_device() == buf._device == dev):
        _scattered("csd_attention", q.get_device(), buf._device, dev)
    rc = _lib().csd_attention(q.data_ptr(), qs[0], qs[1], qs[2], buf.T, buf.q_heads, cache._ref, layer,
                              cache.head_dim ** -0.5 if scale is None else scale, None if n_new is None else _rows_arg(n_new, cache, "n_new"),
                              buf.out.data_ptr(), buf.lse.data_ptr(), buf.workspace.data_ptr(), buf.ws_bytes, _stream_ptr(stream, dev))
    if rc:
        _check(rc, "csd_attention")
    return buf.out
