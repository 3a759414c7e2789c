"""The choice of a beam search's next beams (see ee_beam_select): PyTorch allocates the buffers and provides the stream, libee does the work.

    chosen = select(logits, score, n_beams, end_token=eos, done=done)
    pages.fork(table, chosen.parent.view(-1), group=n_beams, rows=[tokens])        # paged.Pages: the cache goes along
    score, done = chosen.score.view(-1), chosen.done.view(-1)
"""
import struct
from collections import namedtuple

import torch

from . import capi as ee
from .paged import _DTYPES, _keep_derivatives, _number, _refuse, _stream

#: score (float32), parent (a beam of the request; int32), token (int32), each [n_groups][keep]; done (uint8) or None
Selection = namedtuple("Selection", "score parent token done")

_pack_config, _pack_choice = struct.Struct("6i").pack, struct.Struct("PPPP").pack


def selection(n_groups, keep, done=False, device="cuda"):
    """a Selection to be written"""
    make = lambda dtype: torch.empty((n_groups, keep), dtype=dtype, device=device)      # noqa: E731
    return Selection(make(torch.float32), make(torch.int32), make(torch.int32), make(torch.uint8) if done else None)


def workspace(n_groups, n_beams, vocab, keep, device="cuda"):
    """what select needs for these figures, whatever the logits' type; keep one per stream"""
    _number("beams.workspace", n_groups, n_beams, vocab, keep)
    nbytes = ee.load().ee_beam_workspace(_pack_config(n_groups, n_beams, keep, vocab, ee.EE_F32, -1))
    return torch.empty(max(nbytes, 1), dtype=torch.uint8, device=device)


def _of(t, what, shape, dtype, device):
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device or not t.is_contiguous():
        _refuse(f"select: {what} must be a contiguous tensor {tuple(shape)} of {dtype} on device {device}, got {tuple(t.shape)} of {t.dtype} on {t.device}")
    return t.data_ptr()


def select(logits, score, n_beams, *, keep=None, done=None, end_token=-1, out=None, workspace=None):
    """The `keep` (default n_beams) best continuations of each request's n_beams rows of logits [n_groups * n_beams][vocab] (float32 or
    bfloat16, rows at any stride) with running scores `score` (float32 [n_groups * n_beams]; -inf: a beam that is not there).  done (uint8, as
    score): beams that have ended, which go on with end_token at their score.  out: a Selection to write; where keep is n_beams
    its score and done may be those that are read.  The result's done is there if `done` or an end_token is given."""
    if logits.dim() != 2 or logits.dtype not in _DTYPES or (logits.stride(1) != 1 and logits.shape[1] > 1):
        _refuse(f"select: logits must be [rows][vocab] of float32 or bfloat16, contiguous in a row, got {tuple(logits.shape)} of {logits.dtype}")
    keep = n_beams if keep is None else keep
    _number("select", n_beams, keep, end_token)
    rows, vocab = logits.shape
    _number("select", rows, vocab)
    if n_beams < 1 or rows % n_beams:
        _refuse(f"select: {rows} rows are no requests of {n_beams} beams")
    dev = logits.get_device()
    if dev < 0:
        _refuse("select: logits must be on a device")
    _keep_derivatives("select", logits, score)
    n_groups = rows // n_beams
    flat = (rows,)
    if out is None:
        if keep < 1:
            _refuse("select: keep must be positive")
        out = selection(n_groups, keep, done is not None or end_token >= 0, logits.device)
    shape = (n_groups, keep)
    into = _pack_choice(_of(out.score, "out.score", shape, torch.float32, dev), _of(out.parent, "out.parent", shape, torch.int32, dev),
                        _of(out.token, "out.token", shape, torch.int32, dev), 0 if out.done is None else _of(out.done, "out.done", shape, torch.uint8, dev))
    config = _pack_config(n_groups, n_beams, keep, vocab, _DTYPES[logits.dtype], end_token)
    lib = ee.load()
    if workspace is None:
        workspace = torch.empty(max(lib.ee_beam_workspace(config), 1), dtype=torch.uint8, device=logits.device)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        _refuse(f"select: expected a contiguous workspace on device {dev}, got one on {workspace.device}")
    ee.check(lib.ee_beam_select(config, logits.data_ptr(), logits.stride(0), _of(score, "score", flat, torch.float32, dev),
                                None if done is None else _of(done, "done", flat, torch.uint8, dev), into, workspace.data_ptr(), workspace.nbytes, _stream(dev)))
    return out
