"""The end of a fine-tuning step, for many clients at once: each client's own last norm, the frozen vocabulary matrix that all share, and each client's loss, with the gradient that the
backward pass through the layers starts from.  Marshalling only: buffers are torch tensors, all arithmetic happens inside libsymb.so.
"""
from __future__ import annotations

from typing import Dict, Sequence, Tuple

import torch

from . import binding as sb
from .block import _offsets, _on, _workspace

BF16 = torch.bfloat16


class LossHead:
    """x -> loss_i(W norm_i(x)) for the rows of every client i, and the gradient of x.  `norms` hold each client's last norm and where its gradients go, `losses` the scale of its gradient (and its
    temperature, if it learns from a teacher); cap: of the model's logits.  Results are there in the order of the stream given, and stay until the next step."""

    def __init__(self, handle, W: torch.Tensor, lens: Sequence[int], norms: Sequence[sb.Norm], losses: Sequence[sb.Loss], kind: int = sb.SYMB_NORM_RMS, eps: float = 1e-6,
                 weight_base: float = 0.0, reduction: int = sb.SYMB_LOSS_MEAN, cap: float = 0.0):
        if len(norms) != len(lens) or len(losses) != len(lens):
            raise ValueError("one norm and one loss for each client")
        self.h, self.W = handle, W
        vocab, width = W.shape
        off = _offsets(lens)
        self.norm, self.batch = sb.NormBatch(width, off, norms, kind, eps, weight_base), sb.LossBatch(width, vocab, off, losses, reduction, cap)
        self.T, self.width = off[-1], width
        self.N = self.dX = self.loss = self.row_loss = self.ws = None
        self._home: Dict[str, Tuple[int, int]] = {}                    # of each buffer: the stream that it was allocated for, its size

    def _buffer(self, name: str, stream: int, size: int, make) -> torch.Tensor:
        stream_of, room = self._home.get(name, (None, -1))
        if stream_of != stream or room < size:
            with _on(stream):
                setattr(self, name, make())
            self._home[name] = (stream, size)
        return getattr(self, name)

    def _step(self, X: torch.Tensor, taught: Sequence[torch.Tensor], entries: int, gradient: bool, flags: int, stream: int):
        new = lambda *shape, dtype=torch.float32: torch.empty(*shape, device="cuda", dtype=dtype)  # noqa: E731
        need = sb.symb_loss_workspace_bytes(self.batch, entries, gradient)
        if gradient:
            need = max(need, sb.symb_norm_workspace_bytes(self.norm))
        ws = self._buffer("ws", stream, need, lambda: _workspace(need))
        N = self._buffer("N", stream, self.T * self.width, lambda: new(self.T, self.width, dtype=BF16))
        loss, rows = self._buffer("loss", stream, self.batch.S, lambda: new(self.batch.S)), self._buffer("row_loss", stream, self.T, lambda: new(self.T))
        dX = self._buffer("dX", stream, self.T * self.width, lambda: new(self.T, self.width, dtype=BF16)) if gradient else None
        sb.symb_norm_fwd(self.h, self.norm, X, N, stream)
        (sb.symb_distillation if entries else sb.symb_cross_entropy)(self.h, self.batch, N, self.W, *taught, loss, rows, dX, ws, stream)
        if gradient:
            sb.symb_norm_bwd(self.h, self.norm, X, dX, dX, flags, ws, stream)
        return loss, dX

    def cross_entropy(self, X: torch.Tensor, labels: torch.Tensor, gradient: bool = True, flags: int = sb.SYMB_GRAD_OVERWRITE, stream: int = 0):
        """(losses of the clients, gradient of X or None); labels [T] int32, negative ones take no part.  `row_loss` holds the rows' losses; the norms' gradients go to their own tensors."""
        return self._step(X, (labels,), 0, gradient, flags, stream)

    def distillation(self, X: torch.Tensor, ids: torch.Tensor, logits: torch.Tensor, gradient: bool = True, flags: int = sb.SYMB_GRAD_OVERWRITE, stream: int = 0):
        """Likewise, from a teacher's entries: ids [T][entries] int32, negative ones absent, logits [T][entries] fp32."""
        return self._step(X, (ids, logits), ids.shape[1], gradient, flags, stream)
