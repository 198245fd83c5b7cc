"""Between a decoder layer's q/k/v product and its o product: rotary positions,
the paged key/value cache and the attention of new tokens over it (the
`leech_rope`, `leech_cache_*` and `leech_attend` calls of include/leech.h, which
says what each computes and how the cache lies in memory).

Streams: a call runs on `stream`, or on the current one of its tensors' device,
after what that stream holds already: work on other streams that its tensors wait
for is the caller's to order.  Tensors that it allocates (results that no `out` was
given for, workspaces) belong to the stream it runs on.  Tensors handed to a call with
a torch stream may be dropped at once: their memory is not given out again before
that stream has done with it.  Where a stream is named by its handle (an integer or an
ExternalStream, which may end before they do) the caller holds them until it has.
Everything on the device is asynchronous, and may be captured into a graph.
"""
from __future__ import annotations

import math
from contextlib import nullcontext

import numpy as np

from . import _lib

try:
    import torch
except ImportError:          # the host half of the library needs none
    torch = None
else:
    # torch type -> the library's
    _TYPES = {torch.float32: _lib.F32, torch.float16: _lib.F16, torch.bfloat16: _lib.BF16,
              torch.int8: _lib.INT8, torch.float8_e4m3fn: _lib.E4M3}
_HERE = nullcontext()


def _on(device, stream):
    """(context to run a call in, its stream's handle, and the stream if the call's
    tensors have to be kept for it)."""
    if stream is None:
        index = device.index
        handle = torch._C._cuda_getCurrentRawStream(index)
        # (cheaper than torch.cuda.current_device(), which sees to the set-up that a
        # GPU tensor has had)
        if index == torch._C._cuda_getDevice():
            return _HERE, handle, None
        return torch.cuda.device(device), handle, None
    lasting = not isinstance(stream, torch.cuda.ExternalStream)
    if not hasattr(stream, "cuda_stream"):
        handle, lasting = int(stream), False
        # (an ExternalStream of 0 would be a new stream)
        stream = (torch.cuda.ExternalStream(handle, device=device) if handle
                  else torch.cuda.default_stream(device))
    if stream.device != device:
        raise ValueError(f"the stream is on {stream.device}, the tensors on {device}")
    return torch.cuda.stream(stream), stream.cuda_stream, stream if lasting else None


def _keep(stream, *tensors):
    """Keeps the memory of tensors from other uses until `stream` has done with it."""
    for t in tensors:
        if t is not None:
            t.record_stream(stream)


def _new(like, dtype):
    """A contiguous tensor of like's shape and device."""
    if like.is_contiguous():         # half a microsecond less than by shape
        return torch.empty_like(like) if like.dtype == dtype else torch.empty_like(like, dtype=dtype)
    return torch.empty(like.shape, dtype=dtype, device=like.device)


def _gpu(name, t, device=None):
    if not t.is_cuda or (device is not None and t.device != device):
        raise ValueError(f"{name} must be on {device or 'a GPU'}, not on {t.device}")


def _rows(name, x, shape, device):
    """leech_rows of a tensor `shape` = (T, heads, dim) with unit stride along a head."""
    kind = _TYPES.get(x.dtype)
    if kind is None or kind > _lib.BF16 or x.shape != shape:
        raise ValueError(f"{name} must be an f32, f16 or bf16 tensor {list(shape)}, "
                         f"not {x.dtype} {list(x.shape)}")
    ts, hs, ds = x.stride()
    if ds != 1:
        raise ValueError(f"{name} must have unit stride along a head")
    if x.device != device:
        raise ValueError(f"{name} must be on {device}, not on {x.device}")
    return _lib.Rows(x.data_ptr(), kind, ts, hs)


def _index(name, t, dtype, n, device):
    if (t.dtype != dtype or t.dim() != 1 or t.numel() != n or not t.is_contiguous()
            or t.device != device):
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of {n} entries on {device}")
    return t.data_ptr()


# ------------------------------------------------------------------ positions
def rotary_frequencies(width, base=10000.0, scaling=None, factor=1.0, original=None, low=1.0,
                       high=32.0):
    """(radians a position of each of width / 2 pairs as f64, magnitude).

    scaling: None; "linear" (positions divided by `factor`); "ntk" (the base
    grows by factor^(width / (width − 2)), which stretches the slowest pair by
    `factor` and leaves the fastest); "parts" (by frequency, after YaRN,
    arXiv 2309.00071: a pair that turns `high` times or more over the `original`
    length stays, one that turns `low` times or less is stretched by `factor`, a
    line between; the magnitude is 1 + 0.1 ln factor)."""
    if width <= 0 or width % 2:
        raise ValueError("width must be a positive even number")
    if not (base > 0 and factor >= 1 and math.isfinite(base) and math.isfinite(factor)):
        raise ValueError("need a finite base > 0 and a finite factor >= 1")
    i = np.arange(width // 2, dtype=np.float64)
    if scaling == "ntk":
        if width < 4:
            raise ValueError("ntk scaling needs two pairs or more")
        base = base * factor ** (width / (width - 2))
    freq = base ** (-2.0 * i / width)
    if scaling in (None, "ntk"):
        return freq, 1.0
    if scaling == "linear":
        return freq / factor, 1.0
    if scaling == "parts":
        if not original or original <= 0 or not low < high:
            raise ValueError("scaling by parts needs the original length and low < high")
        keep = np.clip((original * freq / (2 * math.pi) - low) / (high - low), 0.0, 1.0)
        return freq * (keep + (1.0 - keep) / factor), 0.1 * math.log(factor) + 1.0
    raise ValueError(f"unknown scaling {scaling!r}")


class Rotary:
    """Rotary positions of the first 2·len(freq) coordinates of a head: freq is
    an f64 device tensor (radians a position of each pair); pairs are (i, i +
    width / 2), or (2i, 2i + 1) when interleaved."""

    def __init__(self, freq, interleaved=False, magnitude=1.0):
        if freq.dtype != torch.float64 or freq.dim() != 1 or not freq.is_contiguous():
            raise ValueError("freq must be a contiguous 1-D f64 tensor")
        self.freq, self.interleaved, self.magnitude = freq, bool(interleaved), float(magnitude)
        self.width, self.device = 2 * freq.numel(), freq.device
        self._c = _lib.RotaryDesc(freq.data_ptr(), self.magnitude, self.width,
                                  int(self.interleaved))

    @classmethod
    def of(cls, width, interleaved=False, device="cuda", **how):
        """From rotary_frequencies(width, **how)."""
        freq, magnitude = rotary_frequencies(width, **how)
        return cls(torch.from_numpy(freq).to(device), interleaved, magnitude)


def rope(x, positions, rotary: Rotary, out=None, dtype=None, transpose=False, stream=None):
    """x [T, heads, dim] (f32, f16 or bf16, any token and head strides) turned by
    positions int64 [T] -> a tensor of `dtype` (x's if None), or `out`, which may
    be x.  transpose: by the opposite angles (the gradient's pass)."""
    if x.dim() != 3:
        raise ValueError("x must be a tensor [T, heads, dim]")
    _gpu("x", x)
    shape, dev = x.shape, x.device
    T, heads, dim = shape
    cx = _rows("x", x, shape, dev)
    pos = _index("positions", positions, torch.int64, T, dev)
    if rotary.device != dev:
        raise ValueError(f"the rotary must be on {dev}, not on {rotary.device}")
    if out is not None and dtype is not None and out.dtype != dtype:
        raise ValueError("out has another dtype than asked for")
    ctx, handle, side = _on(dev, stream)
    with ctx:
        if out is None:
            out = _new(x, dtype or x.dtype)
        _lib.rope(T, heads, dim, cx, pos, rotary._c, transpose, _rows("out", out, shape, dev),
                  handle)
        if side:
            _keep(side, x, positions, rotary.freq, out)
    return out


# ---------------------------------------------------------------------- cache
class KVCache:
    """A paged key/value cache over the caller's tensors: keys [pages, heads,
    page_size, dim] and values [pages, heads, page_size / I, dim, I] (I = 16 /
    bytes of an element) of one dtype, f16, bf16, int8 or float8_e4m3fn, and for
    the 8-bit ones f32 scales [pages, heads, page_size] of each."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        kind = _TYPES.get(k.dtype)
        if kind not in (_lib.F16, _lib.BF16, _lib.INT8, _lib.E4M3) or k.dim() != 4:
            raise ValueError("k must be an f16, bf16, int8 or float8_e4m3fn tensor "
                             "[pages, heads, page_size, dim]")
        pages, heads, page, dim = k.shape
        run = 16 // k.element_size()
        if page % run:
            raise ValueError(f"a page must hold a multiple of {run} tokens")
        if v.dtype != k.dtype or tuple(v.shape) != (pages, heads, page // run, dim, run):
            raise ValueError(f"v must be {k.dtype} [{pages}, {heads}, {page // run}, {dim}, {run}]")
        scales = (k_scale, v_scale) if run == 16 else ()
        if run == 8 and not (k_scale is None and v_scale is None):
            raise ValueError("only 8-bit caches have scales")
        for name, t in zip(("k_scale", "v_scale"), scales):
            if t is None or t.dtype != torch.float32 or tuple(t.shape) != (pages, heads, page):
                raise ValueError(f"{name} must be an f32 tensor [{pages}, {heads}, {page}]")
        for name, t in zip(("k", "v", "k_scale", "v_scale"), (k, v) + scales):
            if not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous")
            _gpu(name, t, k.device)
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.pages, self.heads, self.page_size, self.dim = pages, heads, page, dim
        self.device, self.dtype = k.device, k.dtype
        self._tensors = (k, v, k_scale, v_scale)
        self._c = _lib.KVCacheDesc(kind, heads, dim, page, pages, k.data_ptr(), v.data_ptr(),
                                   *((t.data_ptr() for t in scales) if scales else (None, None)))
        _lib.check_cache(self._c)

    @classmethod
    def empty(cls, pages, page_size, heads, dim, dtype, device="cuda"):
        """A cache of zeros."""
        if dtype not in (torch.float16, torch.bfloat16, torch.int8, torch.float8_e4m3fn):
            raise ValueError("a cache is f16, bf16, int8 or float8_e4m3fn")
        run = 16 // dtype.itemsize
        if page_size % run:
            raise ValueError(f"a page must hold a multiple of {run} tokens")
        k = torch.zeros((pages, heads, page_size, dim), dtype=dtype, device=device)
        v = torch.zeros((pages, heads, page_size // run, dim, run), dtype=dtype, device=device)
        scales = [torch.zeros((pages, heads, page_size), device=device) if run == 16 else None
                  for _ in range(2)]
        return cls(k, v, *scales)

    def write(self, k, v, slots, rotary: Rotary | None = None, positions=None, q=None, out=None,
              dtype=None, stream=None):
        """Keep the tokens k, v [T, heads, dim] (f32, f16 or bf16, any token and
        head strides) in slots int64 [T] (page · page_size + place; out of range:
        not kept; otherwise no two alike), k turned by positions int64 [T] first if a rotary is given.
        With q [T, q_heads, dim], the same launch turns q into `out` (or a new
        tensor of `dtype`, q's if None) and returns it."""
        T, dev = k.shape[0], self.device
        shape = (T, self.heads, self.dim)
        ck, cv = _rows("k", k, shape, dev), _rows("v", v, shape, dev)
        at = _index("slots", slots, torch.int64, T, dev)
        if (rotary is None) != (positions is None):
            raise ValueError("a rotary and positions come together")
        pos = turn = cq = None
        if rotary is not None:
            pos, turn = _index("positions", positions, torch.int64, T, dev), rotary._c
            if rotary.device != dev:
                raise ValueError(f"the rotary must be on {dev}, not on {rotary.device}")
        q_heads = 0
        if q is not None:
            if rotary is None:
                raise ValueError("q is only turned: it needs a rotary")
            if q.dim() != 3 or q.shape[1] == 0:
                raise ValueError("q must be a tensor [T, q_heads, dim]")
            q_heads = q.shape[1]
            q_shape = (T, q_heads, self.dim)
            cq = _rows("q", q, q_shape, dev)
            if out is not None and dtype is not None and out.dtype != dtype:
                raise ValueError("out has another dtype than asked for")
        elif out is not None or dtype is not None:
            raise ValueError("out and dtype are of the turned q")
        ctx, handle, side = _on(dev, stream)
        with ctx:
            if q is not None and out is None:
                out = _new(q, dtype or q.dtype)
            _lib.cache_write(self._c, T, ck, cv, at, pos, turn, q_heads, cq,
                             None if q is None else _rows("out", out, q_shape, dev), handle)
            if side:
                _keep(side, *self._tensors, k, v, slots, positions, rotary and rotary.freq, q, out)
        return out

    def read(self, slots, dtype=None, out=None, stream=None):
        """(k, v) [T, heads, dim] of slots int64 [T] as `dtype` (f16 if None), or
        in the pair `out`; a slot out of range reads as zeros."""
        T = slots.numel()
        at = _index("slots", slots, torch.int64, T, self.device)
        shape = (T, self.heads, self.dim)
        ctx, handle, side = _on(self.device, stream)
        with ctx:
            if out is None:
                out = tuple(torch.empty(shape, dtype=dtype or torch.float16, device=self.device)
                            for _ in range(2))
            elif dtype is not None and any(t.dtype != dtype for t in out):
                raise ValueError("out has another dtype than asked for")
            k, v = out
            ck, cv = _rows("k", k, shape, self.device), _rows("v", v, shape, self.device)
            _lib.cache_read(self._c, T, at, ck, cv, handle)
            if side:
                _keep(side, *self._tensors, slots, k, v)
        return k, v

    def attend(self, q, page_table, kv_len, q_start=None, max_new=None, causal=True, window=0,
               scale=None, out=None, with_lse=False, stream=None):
        """Attention of new tokens over the cache: q [T, q_heads, dim] f16 or bf16
        (16-byte aligned, strides multiples of 8), the new tokens of sequence b in
        rows q_start[b] to q_start[b + 1] (int32 [B + 1]; None: one each, T = B);
        page_table int32 [B, table_pages]; kv_len int32 [B] counts the cached
        tokens, the new ones among them.  max_new: at least every sequence's new
        tokens (None: 1 without q_start, else T; the kernels, launches and workspace go by
        it, so a batch of few new tokens each is quicker with it given).  window > 0: a query sees the last `window` keys up to its
        own.  scale: None for dim^-1/2.  `out` may be q.  Returns out [T, q_heads, dim] of q's type
        (rows of no sequence are not written), and lse f32 [T, q_heads] with
        with_lse."""
        kind = _TYPES.get(q.dtype)
        if kind not in (_lib.F16, _lib.BF16) or q.dim() != 3 or q.shape[2] != self.dim:
            raise ValueError(f"q must be an f16 or bf16 tensor [T, q_heads, {self.dim}]")
        dev = self.device
        T, heads, dim = q.shape
        if page_table.dim() != 2 or page_table.dtype != torch.int32:
            raise ValueError("page_table must be an int32 tensor [B, pages]")
        (B, width), (apart, along) = page_table.shape, page_table.stride()
        if along != 1 and width > 1:
            raise ValueError("page_table must be contiguous along a row")
        if q.device != dev or page_table.device != dev:
            raise ValueError(f"q and page_table must be on {dev}")
        lens = _index("kv_len", kv_len, torch.int32, B, dev)
        starts = None
        if q_start is not None:
            starts = _index("q_start", q_start, torch.int32, B + 1, dev)
        elif T != B:
            raise ValueError("without q_start there is one new token a sequence")
        most = (1 if q_start is None else T) if max_new is None else min(int(max_new), T)
        window = int(window)
        if most < 0 or window < 0:
            raise ValueError("max_new and window must not be negative")
        window = min(window, 0x7FFFFFFF)
        qs = q.stride()
        if qs[2] != 1:
            raise ValueError("q must have unit stride along a head")
        if out is not None and (out.dtype != q.dtype or out.shape != q.shape
                                or out.stride(2) != 1 or out.device != dev):
            raise ValueError("out must have q's type, shape and device and unit stride along a head")
        ctx, handle, side = _on(dev, stream)
        with ctx:
            if out is None:
                out = _new(q, q.dtype)
            os_ = out.stride()
            lse = torch.empty((T, heads), dtype=torch.float32, device=dev) if with_lse else None
            args = _lib.AttendArgs(
                kind, heads, T, q.data_ptr(), qs[0], qs[1], out.data_ptr(), os_[0], os_[1],
                lse.data_ptr() if with_lse else None, B, starts, lens, page_table.data_ptr(),
                apart, width, most, int(causal), window,
                dim ** -0.5 if scale is None else scale, None, 0)
            size = _lib.attend_workspace(self._c, args)
            if size:
                room = torch.empty(size, dtype=torch.uint8, device=dev)
                args.workspace, args.workspace_bytes = room.data_ptr(), size
            _lib.attend(self._c, args, handle)
            if side:
                _keep(side, *self._tensors, q, page_table, kv_len, q_start, out)
        return (out, lse) if with_lse else out
