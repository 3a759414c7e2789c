"""Device-memory plumbing around libee's rotary tables and paged cache: PyTorch allocates the buffers and provides the
stream, libee does all the work.  What a server does with them, per layer and step:

    rope = Rope(head_dim, max_pos)
    kv = PagedCache(n_layers, n_pages, n_kv_heads, head_dim, page_size, dtype="bf16")
    step = PagedStep(q_start, kv_len, pages, n_tokens=, max_q_len=, max_kv_len=)
    append(kv, layer, step, k, v, rope=rope, q=q, q_out=q)
    out = attend(kv, layer, step, q)
"""
import ctypes as C

import torch

from . import capi as ee
from .session import _ptr, _stream

_PAIRINGS = {"half": ee.EE_ROPE_HALF, "interleaved": ee.EE_ROPE_INTERLEAVED}
_SCALINGS = {"none": ee.EE_ROPE_UNSCALED, "linear": ee.EE_ROPE_LINEAR, "base": ee.EE_ROPE_BASE, "bands": ee.EE_ROPE_BANDS}
_DTYPES = {torch.float32: ee.EE_F32, torch.bfloat16: ee.EE_BF16}


def _refuse(what):
    raise ee.EEError(ee.EE_ERR_INVALID_ARG, what)


def _heads(t, what, n_tokens, n_heads, hd, dtype):
    """ee_heads of a tensor [n_tokens][n_heads][hd] whose features are contiguous"""
    if tuple(t.shape) != (n_tokens, n_heads, hd) or t.dtype != dtype or not t.is_cuda:
        _refuse(f"{what}: expected a device tensor {(n_tokens, n_heads, hd)} of {dtype}, got {tuple(t.shape)} of {t.dtype} on {t.device}")
    st = t.stride()
    if st[2] != 1 and hd > 1:
        _refuse(f"{what}: the features of a head must be contiguous")
    return ee.ee_heads(t.data_ptr(), st[0], st[1])


def _int32(t, what, n):
    """a contiguous int32 device tensor of n values"""
    if t.dtype != torch.int32 or not t.is_cuda or not t.is_contiguous() or t.numel() != n:
        _refuse(f"{what}: expected a contiguous int32 device tensor of {n} values, got {t.numel()} of {t.dtype} on {t.device}")
    return t


class Rope:
    """A rotary table (see ee_rope_config): rot_dim features of a head turn (default: all), in "half" or "interleaved" pairs,
    at frequencies scaled by "none", "linear", "base" or "bands"."""

    def __init__(self, head_dim, max_pos, *, rot_dim=None, pairing="half", theta=10000.0, scaling="none", factor=1.0, trained_pos=0,
                 low=1.0, high=4.0, magnitude=0.0):
        if pairing not in _PAIRINGS or scaling not in _SCALINGS:
            _refuse(f"Rope: unknown pairing {pairing!r} or scaling {scaling!r}")
        self.lib = ee.load()
        self.cfg = ee.ee_rope_config(head_dim, head_dim if rot_dim is None else rot_dim, _PAIRINGS[pairing], max_pos, _SCALINGS[scaling],
                                     trained_pos, theta, factor, low, high, magnitude)
        self.h = C.c_void_p()
        ee.check(self.lib.ee_rope_create(C.byref(self.cfg), C.byref(self.h)))

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
        """x [n][heads][head_dim] (float32 or bfloat16, any token and head stride) rotated at pos (int32 [n]); out may be x.
        inverse: by the negative angle, which is the gradient with respect to x of a result's gradient."""
        if x.dim() != 3 or x.dtype not in _DTYPES:
            _refuse(f"Rope.apply: x must be [tokens][heads][features] of float32 or bfloat16, got {tuple(x.shape)} of {x.dtype}")
        n, heads, hd = x.shape
        if out is None:
            out = torch.empty((n, heads, hd), dtype=x.dtype, device=x.device)
        xh, yh = (_heads(t, "Rope.apply", n, heads, self.cfg.head_dim, x.dtype) for t in (x, out))
        ee.check(self.lib.ee_rope_apply(self.h, _DTYPES[x.dtype], C.byref(xh), C.byref(yh), _ptr(_int32(pos, "Rope.apply: pos", n)), n, heads,
                                        int(inverse), None if status is None else _ptr(_int32(status, "Rope.apply: status", 1)), _stream()))
        return out


class PagedCache:
    """A pool of pages (see ee_paged_config) and its allocation; .pool is the whole pool, flat, in the cache's type."""

    def __init__(self, n_layers, n_pages, n_kv_heads, head_dim, page_size, dtype="bf16"):
        self.lib = ee.load()
        self.cfg = ee.ee_paged_config(n_layers, n_pages, n_kv_heads, head_dim, page_size, ee.EE_BF16 if dtype == "bf16" else ee.EE_F32)
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        nbytes = self.lib.ee_paged_pool_bytes(C.byref(self.cfg))
        if nbytes == 0:
            raise ee.EEError(ee.EE_ERR_SHAPE, self.lib.ee_last_error().decode())
        self.pool = torch.empty(nbytes // self.dtype.itemsize, dtype=self.dtype, device="cuda")
        self.h = C.c_void_p()
        ee.check(self.lib.ee_paged_bind(C.byref(self.cfg), _ptr(self.pool), nbytes, C.byref(self.h)))

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
        nbytes = self.lib.ee_paged_attention_workspace(self.h, n_q_heads, C.byref(step.c))
        return torch.empty(max(nbytes, 1), dtype=torch.uint8, device="cuda")


class PagedStep:
    """The new rows of one call (see ee_paged_step).  q_start [n_seqs + 1], kv_len [n_seqs] and pages [n_seqs][width] are int32
    device tensors that the calls read when they run, so a recorded graph sees what they hold at each replay; status (int32 [1])
    collects refusals."""

    def __init__(self, q_start, kv_len, pages, *, n_tokens, max_q_len, max_kv_len, status=None):
        n = kv_len.numel()
        if pages.dim() != 2 or pages.shape[0] != n:
            _refuse(f"PagedStep: pages must be [{n}][pages per sequence], got {tuple(pages.shape)}")
        self.tensors = (_int32(q_start, "PagedStep: q_start", n + 1), _int32(kv_len, "PagedStep: kv_len", n),
                        _int32(pages, "PagedStep: pages", pages.numel()), None if status is None else _int32(status, "PagedStep: status", 1))
        self.c = ee.ee_paged_step(n, n_tokens, max_q_len, max_kv_len, pages.shape[1], *(None if t is None else t.data_ptr() for t in self.tensors))
        self.n_tokens = n_tokens


def append(kv, layer, step, k, v, *, rope=None, q=None, q_out=None):
    """Keys (rotated by rope) and values [n_tokens][n_kv_heads][head_dim] to the rows' positions of `layer`; with q
    [n_tokens][n_q_heads][head_dim] also the rotated queries to q_out (default: a new tensor, which is returned)."""
    n, c = step.n_tokens, kv.cfg
    kh, vh = (_heads(t, "append", n, c.n_kv_heads, c.head_dim, kv.dtype) for t in (k, v))
    qh = qo = None
    n_q = 0
    if q is not None:
        n_q = q.shape[1]
        if q_out is None:
            q_out = torch.empty((n, n_q, c.head_dim), dtype=q.dtype, device=q.device)
        qh, qo = (_heads(t, "append", n, n_q, c.head_dim, kv.dtype) for t in (q, q_out))
        qh, qo = C.byref(qh), C.byref(qo)
    ee.check(kv.lib.ee_paged_append(kv.h, layer, C.byref(step.c), None if rope is None else rope.h, C.byref(kh), C.byref(vh), qh, qo, n_q,
                                    _stream()))
    return q_out


def attend(kv, layer, step, q, *, out=None, scale=None, window=0, workspace=None):
    """Attention of the step's rows q [n_tokens][n_q_heads][head_dim] over the cached positions of `layer`; scale defaults to
    1/sqrt(head_dim), window 0 is all earlier positions, workspace is kv.workspace's."""
    n, c = step.n_tokens, kv.cfg
    if q.dim() != 3:
        _refuse(f"attend: q must be [tokens][heads][features], got {tuple(q.shape)}")
    heads = q.shape[1]
    if out is None:
        out = torch.empty((n, heads, c.head_dim), dtype=kv.dtype, device=q.device)
    if workspace is None:
        workspace = kv.workspace(step, heads)
    qh, oh = (_heads(t, "attend", n, heads, c.head_dim, kv.dtype) for t in (q, out))
    ee.check(kv.lib.ee_paged_attention(kv.h, layer, C.byref(step.c), C.byref(qh), C.byref(oh), heads,
                                       c.head_dim ** -0.5 if scale is None else scale, window, _ptr(workspace), workspace.numel(), _stream()))
    return out
