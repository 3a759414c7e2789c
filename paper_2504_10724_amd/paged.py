"""Device-memory plumbing around libee's rotary tables, paged cache and its pages' bookkeeping: PyTorch allocates the buffers and provides
the stream, libee does all the work.  What a server does with them, per layer and step (examples/paged_serving.py runs it):

    rope = Rope(head_dim, max_pos)
    kv = PagedCache(n_layers, n_pages, n_kv_heads, head_dim, page_size, dtype="bf16")
    step = PagedStep(q_start, kv_len, pages, n_tokens=, max_q_len=, max_kv_len=)
    append(kv, layer, step, k, v, rope=rope, q=q, q_out=q)
    out = attend(kv, layer, step, q)

Who owns which page is the server's own business there; where what decides about it is on the device, as in a beam search, the pages
are kept there too (examples/beam_search.py):

    pages, table = Pages(kv, max_seqs), PageTable(kv, n_seqs, pages_per_seq)
    pages.fork(table, parent, group=n_beams, rows=[tokens])
    pages.grow(table)
    step = PagedStep(q_start, table.kv_len, table.pages, n_tokens=, max_q_len=, max_kv_len=)
"""
import ctypes as C
import struct

import torch
from torch.autograd import forward_ad

from . import capi as ee
from .session import _raw_stream

_PAIRINGS = {"half": ee.EE_ROPE_HALF, "interleaved": ee.EE_ROPE_INTERLEAVED}
_SCALINGS = {"none": ee.EE_ROPE_UNSCALED, "linear": ee.EE_ROPE_LINEAR, "base": ee.EE_ROPE_BASE, "bands": ee.EE_ROPE_BANDS}
_DTYPES = {torch.float32: ee.EE_F32, torch.bfloat16: ee.EE_BF16}


def _refuse(what):
    raise ee.EEError(ee.EE_ERR_INVALID_ARG, what)


_stream_of = _raw_stream or (lambda device: torch.cuda.current_stream(device).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream(device):
    """Handle of the current stream of a device, by its number (a fifth of the time the way through the current device takes).  A default
    stream's handle is 0 on every device and means the current one's: work for another device's memory would go there."""
    handle = _stream_of(device)
    if not handle and _current_device() != device:
        _refuse(f"tensors are on device {device}, whose stream is its default one, but device {_current_device()} is current: use torch.cuda.device({device})")
    return handle


_MOST = 2 ** 31 - 1


def _number(what, *values):
    """the library's counts have 32 bits, and the binding would pass on the lowest 32 of a larger one"""
    for v in values:
        if not -_MOST <= v <= _MOST:
            _refuse(f"{what}: {v} does not fit 32 bits")


_pack_heads = struct.Struct("Pqq").pack      # an ee_heads as bytes, a fifth of the time a ctypes structure takes


def _heads(t, what, shape, dtype, device, written=False):
    """ee_heads of a tensor [n_tokens][n_heads][hd] on device number `device` whose features are contiguous; of one that is written, no
    two rows or heads in one place"""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device:
        _refuse(f"{what}: expected a tensor {tuple(shape)} of {dtype} on device {device}, got {tuple(t.shape)} of {t.dtype} on {t.device}")
    token, head, feature = t.stride()
    if feature != 1 and shape[2] > 1:
        _refuse(f"{what}: the features of a head must be contiguous")
    if written and not (token and head) and ((token == 0 and shape[0] > 1) or (head == 0 and shape[1] > 1)):
        _refuse(f"{what}: rows or heads of the result share their memory")
    return _pack_heads(t.data_ptr(), token, head)


def _int32(t, what, n, device):
    """a contiguous int32 tensor of n values on device number `device`"""
    if t.dtype is not torch.int32 or t.numel() != n or t.get_device() != device or device < 0 or not t.is_contiguous():
        _refuse(f"{what}: expected a contiguous int32 tensor of {n} values on a device ({device}), got {t.numel()} of {t.dtype} on {t.device}")
    return t


def _keep_derivatives(what, *tensors):
    """The operator has no gradient, and a result that the caller provides takes no part in a graph: where a tensor needs one, or carries the
    tangent of a forward-mode derivative (no_grad leaves those on), the call is refused and nothing gets lost."""
    if torch.is_grad_enabled():
        for t in tensors:
            if t.requires_grad:
                _refuse(f"{what}: a tensor requires a gradient that is not computed; call it under torch.no_grad() or on detached tensors")
    if getattr(forward_ad, "_current_level", 0) >= 0 and any(forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        _refuse(f"{what}: a tensor carries a forward-mode gradient that is not computed; call it on detached tensors")


class _Turn(torch.autograd.Function):
    """Rope.apply in a graph: its gradient is the inverse rotation of the result's.  Rows that are left out are zeros both ways."""

    @staticmethod
    def forward(ctx, x, pos, rope, inverse, status):
        ctx.save_for_backward(pos)
        ctx.rope, ctx.inverse = rope, inverse
        return rope.apply(x, pos, out=torch.zeros(x.shape, dtype=x.dtype, device=x.device), inverse=inverse, status=status)

    @staticmethod
    def backward(ctx, g):
        g = g if g.stride(2) == 1 else g.contiguous()
        return _Turn.apply(g, *ctx.saved_tensors, ctx.rope, not ctx.inverse, None), None, None, None, None


class Rope:
    """A rotary table (see ee_rope_config): rot_dim features of a head turn (default: all), in "half" or "interleaved" pairs,
    at frequencies scaled by "none", "linear", "base" or "bands"."""

    def __init__(self, head_dim, max_pos, *, rot_dim=None, pairing="half", theta=10000.0, scaling="none", factor=1.0, trained_pos=0,
                 low=1.0, high=4.0, magnitude=0.0):
        if pairing not in _PAIRINGS or scaling not in _SCALINGS:
            _refuse(f"Rope: unknown pairing {pairing!r} or scaling {scaling!r}")
        _number("Rope", head_dim, max_pos, 0 if rot_dim is None else rot_dim, trained_pos)
        self.lib = ee.load()
        self.cfg = ee.ee_rope_config(head_dim, head_dim if rot_dim is None else rot_dim, _PAIRINGS[pairing], max_pos, _SCALINGS[scaling],
                                     trained_pos, theta, factor, low, high, magnitude)
        self.h = C.c_void_p()
        ee.check(self.lib.ee_rope_create(C.byref(self.cfg), C.byref(self.h)))
        self.device = torch.cuda.current_device()            # where the table is

    def close(self):
        if self.h:
            self.lib.ee_rope_destroy(self.h)
            self.h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def apply(self, x, pos, *, out=None, inverse=False, status=None):
        """x [n][heads][head_dim] (float32 or bfloat16, any token and head stride, on the table's device) rotated at pos (int32 [n]);
        out may be x.  A row whose position is outside the table is not written: without `out` it holds what the new tensor's memory held.
        inverse: by the negative angle, which is the gradient with respect to x of a result's gradient.  Where x requires a gradient the
        result has it, and rows outside the table are zeros; `out` is refused there."""
        dtype, shape = x.dtype, x.shape
        if len(shape) != 3 or dtype not in _DTYPES or shape[2] != self.cfg.head_dim:
            _refuse(f"Rope.apply: x must be [tokens][heads][{self.cfg.head_dim}] of float32 or bfloat16, got {tuple(shape)} of {dtype}")
        if out is not None:
            _keep_derivatives("Rope.apply with out", x, out)
        elif x.requires_grad and torch.is_grad_enabled():
            return _Turn.apply(x, pos, self, inverse, status)
        else:
            _keep_derivatives("Rope.apply", x)
            out = torch.empty(shape, dtype=dtype, device=x.device)
        n, heads, _ = shape
        dev = self.device
        ee.check(self.lib.ee_rope_apply(self.h, _DTYPES[dtype], _heads(x, "Rope.apply", shape, dtype, dev),
                                        _heads(out, "Rope.apply", shape, dtype, dev, True), _int32(pos, "Rope.apply: pos", n, dev).data_ptr(), n, heads,
                                        inverse, None if status is None else _int32(status, "Rope.apply: status", 1, dev).data_ptr(), _stream(dev)))
        return out


class PagedCache:
    """A pool of pages (see ee_paged_config) and its allocation; .pool is the whole pool, flat, in the cache's type."""

    def __init__(self, n_layers, n_pages, n_kv_heads, head_dim, page_size, dtype="bf16"):
        if dtype not in ("bf16", "f32"):
            raise ee.EEError(ee.EE_ERR_DTYPE, f"PagedCache: unknown dtype {dtype!r}")
        _number("PagedCache", n_layers, n_pages, n_kv_heads, head_dim, page_size)
        self.lib = ee.load()
        self.cfg = ee.ee_paged_config(n_layers, n_pages, n_kv_heads, head_dim, page_size, ee.EE_BF16 if dtype == "bf16" else ee.EE_F32)
        self.dtype, self.n_kv_heads, self.head_dim = (torch.bfloat16 if dtype == "bf16" else torch.float32), n_kv_heads, head_dim
        nbytes = self.lib.ee_paged_pool_bytes(C.byref(self.cfg))
        if nbytes == 0:
            raise ee.EEError(ee.EE_ERR_SHAPE, self.lib.ee_last_error().decode())
        self.pool = torch.empty(nbytes // self.dtype.itemsize, dtype=self.dtype, device="cuda")
        self.scale, self.device = head_dim ** -0.5, self.pool.get_device()
        self.h = C.c_void_p()
        ee.check(self.lib.ee_paged_bind(C.byref(self.cfg), self.pool.data_ptr(), nbytes, C.byref(self.h)))

    def close(self):
        if self.h:
            self.lib.ee_paged_destroy(self.h)
            self.h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def workspace(self, step, n_q_heads):
        """what attend needs for this step and every step whose host figures are at most its; keep one per stream"""
        nbytes = self.lib.ee_paged_attention_workspace(self.h, n_q_heads, step.ref)
        return torch.empty(max(nbytes, 1), dtype=torch.uint8, device=self.pool.device)


class PagedStep:
    """The new rows of one call (see ee_paged_step).  q_start [n_seqs + 1], kv_len [n_seqs] and pages [n_seqs][width] are int32
    tensors on the cache's device that the calls read when they run, so a recorded graph sees what they hold at each replay; status
    (int32 [1]) collects refusals."""

    def __init__(self, q_start, kv_len, pages, *, n_tokens, max_q_len, max_kv_len, status=None):
        n = kv_len.numel()
        if pages.dim() != 2 or pages.shape[0] != n:
            _refuse(f"PagedStep: pages must be [{n}][pages per sequence], got {tuple(pages.shape)}")
        _number("PagedStep", n_tokens, max_q_len, max_kv_len)
        self.device = dev = kv_len.get_device()
        self.tensors = (_int32(q_start, "PagedStep: q_start", n + 1, dev), _int32(kv_len, "PagedStep: kv_len", n, dev),
                        _int32(pages, "PagedStep: pages", pages.numel(), dev),
                        None if status is None else _int32(status, "PagedStep: status", 1, dev))
        self.c = ee.ee_paged_step(n, n_tokens, max_q_len, max_kv_len, pages.shape[1], *(None if t is None else t.data_ptr() for t in self.tensors))
        self.n_tokens, self.ref = n_tokens, C.byref(self.c)


def append(kv, layer, step, k, v, *, rope=None, q=None, q_out=None):
    """Keys (rotated by rope) and values [n_tokens][n_kv_heads][head_dim] to the rows' positions of `layer`; with q
    [n_tokens][n_q_heads][head_dim] also the rotated queries to q_out (default: a new tensor, which is returned; rows that are left out
    hold what its memory held).  Everything is on the cache's device."""
    dtype, shape, dev = kv.dtype, (step.n_tokens, kv.n_kv_heads, kv.head_dim), kv.device
    if step.device != dev or (rope is not None and rope.device != dev):
        _refuse(f"append: the step or the rotary table is not on the cache's device ({dev})")
    if rope is not None and not rope.h:                      # the library takes no table for no rotation
        _refuse("append: the rotary table is closed")
    if not -_MOST <= layer <= _MOST:
        _number("append", layer)
    _keep_derivatives("append", k, v)
    kh, vh = _heads(k, "append", shape, dtype, dev), _heads(v, "append", shape, dtype, dev)
    qh = qo = None
    n_q = 0
    if q is not None:
        n_q = q.shape[1]
        shape = (step.n_tokens, n_q, kv.head_dim)
        if q_out is None:
            q_out = torch.empty(shape, dtype=dtype, device=q.device)
        _keep_derivatives("append", q, q_out)
        qh, qo = _heads(q, "append", shape, dtype, dev), _heads(q_out, "append", shape, dtype, dev, True)
    ee.check(kv.lib.ee_paged_append(kv.h, layer, step.ref, None if rope is None else rope.h, kh, vh, qh, qo, n_q, _stream(dev)))
    return q_out


def attend(kv, layer, step, q, *, out=None, scale=None, window=0, workspace=None):
    """Attention of the step's rows q [n_tokens][n_q_heads][head_dim] over the cached positions of `layer`; scale defaults to
    1/sqrt(head_dim), window 0 is all earlier positions, workspace is kv.workspace's.  Everything is on the cache's device.  Rows of
    a sequence outside the step's figures are not written: without `out` they hold what the new tensor's memory held."""
    if q.dim() != 3:
        _refuse(f"attend: q must be [tokens][heads][features], got {tuple(q.shape)}")
    heads = q.shape[1]
    shape, dtype, dev = (step.n_tokens, heads, kv.head_dim), kv.dtype, kv.device
    if step.device != dev:
        _refuse(f"attend: the step is not on the cache's device ({dev})")
    if not (-_MOST <= layer <= _MOST and -_MOST <= window <= _MOST):
        _number("attend", layer, min(window, _MOST))
        window = _MOST                                       # wider than any sequence
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=q.device)
    _keep_derivatives("attend", q, out)
    if workspace is None:
        workspace = kv.workspace(step, heads)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        _refuse(f"attend: expected a contiguous workspace on device {dev}, got one on {workspace.device}")
    ee.check(kv.lib.ee_paged_attention(kv.h, layer, step.ref, _heads(q, "attend", shape, dtype, dev), _heads(out, "attend", shape, dtype, dev, True),
                                       heads, kv.scale if scale is None else scale, window, workspace.data_ptr(), workspace.nbytes,
                                       _stream(dev)))
    return out


class PageTable:
    """A table of pages (see ee_page_table), empty: pages [n_seqs][pages_per_seq] and kv_len [n_seqs], int32 on the cache's device, which
    PagedStep takes as they are and Pages alone changes."""

    def __init__(self, kv, n_seqs, pages_per_seq):
        _number("PageTable", n_seqs, pages_per_seq)
        if n_seqs < 0 or pages_per_seq < 0:
            _refuse("PageTable: negative count")
        self.device = kv.device
        self.pages = torch.full((n_seqs, pages_per_seq), -1, dtype=torch.int32, device=kv.pool.device)
        self.kv_len = torch.zeros(n_seqs, dtype=torch.int32, device=kv.pool.device)
        self.c = ee.ee_page_table(n_seqs, pages_per_seq, self.pages.data_ptr(), self.kv_len.data_ptr())
        self.n_seqs, self.ref = n_seqs, C.byref(self.c)


_pack_rows = struct.Struct("Pqq").pack


class Pages:
    """Who holds which page of a cache (see ee_pages_*), all of them free; tables of up to max_seqs rows grow.  refs (int32 [n_pages])
    counts the entries that name a page: pages.refs == 0 are the free ones.  Calls change the tables in place and return nothing;
    status (int32 [1]) collects refusals."""

    def __init__(self, kv, max_seqs):
        _number("Pages", max_seqs)
        self.lib, self.kv, self.device = kv.lib, kv, kv.device
        if not kv.h:
            _refuse("Pages: the cache is closed")
        nbytes = self.lib.ee_pages_state_bytes(kv.h, max_seqs)
        self.state = torch.empty(nbytes, dtype=torch.uint8, device=kv.pool.device)
        self.refs = self.state[:4 * kv.cfg.n_pages].view(torch.int32)
        self.h = C.c_void_p()
        ee.check(self.lib.ee_pages_bind(kv.h, max_seqs, self.state.data_ptr() or 256, nbytes, C.byref(self.h)))
        self.reset()

    def close(self):
        if self.h:
            self.lib.ee_pages_destroy(self.h)
            self.h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, what, *tables):
        if not self.kv.h:                                    # the library's handle would look into it
            _refuse(f"{what}: the cache is closed")
        for t in tables:
            if t.device != self.device:
                _refuse(f"{what}: a table is not on the cache's device ({self.device})")

    def _ints(self, t, what, n):
        return None if t is None else _int32(t, what, n, self.device).data_ptr()

    def reset(self):
        """every page is free; tables that name some are the caller's to clear"""
        self._check("Pages.reset")
        ee.check(self.lib.ee_pages_reset(self.h, _stream(self.device)))

    def grow(self, table, new=None, *, status=None):
        """new (int32 [n_seqs], default one each) positions more for the table's rows; pages that others hold too are copied before they
        are written"""
        self._check("Pages.grow", table)
        ee.check(self.lib.ee_pages_grow(self.h, table.ref, self._ints(new, "Pages.grow: new", table.n_seqs),
                                        self._ints(status, "Pages.grow: status", 1), _stream(self.device)))

    def fork(self, table, parent, *, source=None, keep=None, group=0, rows=(), status=None):
        """Row i of the table becomes row parent[i] (int32; -1: empty) of source (default: the table itself, in place), cut to keep[i]
        positions; with `group`, parents are numbered inside groups of that many rows.  rows: tensors [n_seqs][...] whose rows go along."""
        self._check("Pages.fork", table, *(() if source is None else (source,)))
        _number("Pages.fork", group)
        packed, rows = [], tuple(rows)
        if rows:
            _keep_derivatives("Pages.fork", *rows)
        for x in rows:
            if x.dim() < 1 or x.shape[0] != table.n_seqs or x.get_device() != self.device or not (x.is_contiguous() or x[0].is_contiguous()):
                _refuse(f"Pages.fork: rows must be [{table.n_seqs}][...] on device {self.device}, each row contiguous, got {tuple(x.shape)} on {x.device}")
            size = x.element_size()
            packed.append(_pack_rows(x.data_ptr(), x.stride(0) * size, x.numel() // max(table.n_seqs, 1) * size))
        ee.check(self.lib.ee_pages_fork(self.h, table.ref, None if source is None else source.ref, self._ints(parent, "Pages.fork: parent", table.n_seqs),
                                        self._ints(keep, "Pages.fork: keep", table.n_seqs), group, b"".join(packed) or None, len(packed),
                                        self._ints(status, "Pages.fork: status", 1), _stream(self.device)))

    def compact(self, *tables):
        """the pages in use move to the lowest numbers; tables: all that name pages of this cache"""
        self._check("Pages.compact", *tables)
        ee.check(self.lib.ee_pages_compact(self.h, b"".join(bytes(t.c) for t in tables) or None, len(tables), _stream(self.device)))


def copy_pages(source, to, from_pages, to_pages, *, status=None):
    """page from_pages[i] of the cache `source` to page to_pages[i] of the cache `to` (int32), in all layers"""
    if source.device != to.device:
        _refuse(f"copy_pages: caches on different devices ({source.device}, {to.device})")
    n, dev = from_pages.numel(), source.device
    ee.check(source.lib.ee_pages_copy(source.h, to.h, _int32(from_pages, "copy_pages", n, dev).data_ptr(), _int32(to_pages, "copy_pages", n, dev).data_ptr(),
                                      n, None if status is None else _int32(status, "copy_pages: status", 1, dev).data_ptr(), _stream(dev)))
