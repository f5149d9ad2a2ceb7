"""Beam search's choice over beams and vocabulary for PyTorch users: tensors and streams are torch's, all work runs in
libtss.so (tss_beam_*).

``BeamSelector.select`` picks every group's best continuations on the device; its ``parent`` is what
``paged.PagePool.reorder`` takes to move the beams' pages, without a host wait between the two (64 sequences a call: of more
rows, each call gets the parents of its texts less its first row's number).  All tensors are on the
selector's GPU, which has to be the current device in every call.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import native
from .native import _P, check, lib
from .paged import _code, _stream_of


class BeamSelector:
    """Workspace for up to `rows` rows of `vocab` logits and up to `keep` continuations of a group, on the current device (or
    `device`)."""

    def __init__(self, rows: int, vocab: int, keep: int, device: Optional[int] = None):
        self._dev = torch.cuda.current_device() if device is None else device
        self.rows, self.vocab, self.keep = rows, vocab, keep
        self._c_select = lib().tss_beam_select
        h = _P()
        with torch.cuda.device(self._dev):
            check(lib().tss_beam_create(rows, vocab, keep, ctypes.byref(h)), "tss_beam_create")
        self._h = h

    def close(self) -> None:
        if getattr(self, "_h", None):
            lib().tss_beam_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _of(self, t: torch.Tensor, shape, dtype, what: str) -> int:
        if t.shape != shape or t.dtype != dtype or not t.is_contiguous() or t.get_device() != self._dev:
            raise ValueError(f"{what}: contiguous {dtype} {list(shape)} on the selector's GPU is wanted")
        return t.data_ptr()

    def select(self, logits: torch.Tensor, score: Optional[torch.Tensor], score_out: torch.Tensor, parent: torch.Tensor,
               token: torch.Tensor, *, n_beams: int, done: Optional[torch.Tensor] = None, end_token: int = 0, stream=None) -> None:
        """The best continuations of every n_beams rows of logits [rows][vocab] (any stride between rows) after beams of the values
        score (float32 [rows]; None: zeros): score_out float32, parent (a row of logits) and token int32 [groups][kept].  done:
        int32 [rows], not 0 for finished beams, which go on with end_token and their score; None: none is."""
        if logits.dim() != 2 or logits.get_device() != self._dev or logits.shape[1] != self.vocab or (logits.shape[0] and logits.stride(1) != 1):
            raise ValueError("logits: [rows][vocab] on the selector's GPU, a row's contiguous, is wanted")
        rows, i32 = logits.shape[0], torch.int32
        if n_beams < 1 or rows % n_beams or score_out.dim() != 2:
            raise ValueError("groups of n_beams rows and score_out [groups][kept] are wanted")
        shape = (rows // n_beams, score_out.shape[1])
        a = native.TssBeamArgs(shape[0], n_beams, shape[1], _code(logits), logits.data_ptr(), logits.stride(0) if rows > 1 else self.vocab,
                               None if score is None else self._of(score, (rows,), torch.float32, "score"),
                               None if done is None else self._of(done, (rows,), i32, "done"), end_token,
                               self._of(score_out, shape, torch.float32, "score_out"), self._of(parent, shape, i32, "parent"),
                               self._of(token, shape, i32, "token"))
        s = self._c_select(self._h, ctypes.byref(a), _stream_of(self._dev, stream))
        if s:
            check(s, "tss_beam_select")

    def sync_status(self, stream=None) -> int:
        return lib().tss_beam_sync_status(self._h, _stream_of(self._dev, stream))
