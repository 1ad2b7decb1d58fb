"""Losses over the vocabulary on hidden rows and an LM head, with their gradients: cross entropy of given tokens and distillation from a teacher's top logits.

The binding of tr_cross_entropy, tr_distill and their gradients (include/tokroute.h states what they compute, which rows count, and how types go together).
A `VocabLoss` keeps the workspace that calls share; `cross_entropy` and `distill` are the same losses for programs that differentiate with autograd.
There is no CPU fallback: without the built library or without a GPU calls raise.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import tokroute
from .tokroute import TokrouteError, tr_loss_config, tr_loss_grads, tr_loss_rows

_DTYPES = {torch.float32: tokroute.F32, torch.bfloat16: tokroute.BF16}


class VocabLoss:
    """Workspace and sizes of loss calls: up to max_rows hidden rows of `dim` features, a head of `vocab` entries, up to max_entries teacher entries a row.

    Calls enqueue on the current stream of `device`, whichever device is current; calls of one VocabLoss on different streams must be ordered by the caller, since they share the workspace.
    Hidden rows and heads may be strided from row to row; each row is contiguous.
    """

    def __init__(self, max_rows: int, dim: int, vocab: int, hidden_dtype=torch.bfloat16, weight_dtype=torch.bfloat16, max_entries: int = 1, device="cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("tokroute needs a GPU: no CPU path exists")
        if hidden_dtype not in _DTYPES or weight_dtype not in _DTYPES:
            raise ValueError(f"hidden rows and heads are float32 or bfloat16, not {hidden_dtype} and {weight_dtype}")
        self.lib = tokroute.load_library()
        self.device = torch.device(device)
        self.hidden_dtype, self.weight_dtype = hidden_dtype, weight_dtype
        self.cfg = tr_loss_config(max_rows, dim, vocab, _DTYPES[hidden_dtype], _DTYPES[weight_dtype], max_entries)
        nbytes = self.lib.tr_loss_workspace_bytes(C.byref(self.cfg))
        if nbytes == 0:
            raise TokrouteError(tokroute.ERR_SHAPE, "tr_loss_workspace_bytes", "(sizes or types not supported)")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        self._home = torch.cuda.current_stream(self.device)

    # -- helpers
    def _stream(self):
        s = torch.cuda.current_stream(self.device)
        if s != self._home:
            self.workspace.record_stream(s)    # its memory is not handed on while work of that stream may use it
        return s.cuda_stream

    def _matrix(self, t, what, dtype, cols, rows=None):
        if not (isinstance(t, torch.Tensor) and t.is_cuda and t.device == self.workspace.device and t.dtype == dtype and t.dim() == 2 and t.shape[1] == cols
                and (rows is None or t.shape[0] == rows) and (t.stride(1) == 1 or cols == 1)):
            raise ValueError(f"{what}: a {dtype} matrix of {cols} columns{'' if rows is None else f' and {rows} rows'} with contiguous rows on {self.workspace.device}")
        return max(t.stride(0), cols) if t.shape[0] <= 1 else t.stride(0)

    def _flat(self, t, what, dtype, shape):
        if not (isinstance(t, torch.Tensor) and t.is_cuda and t.device == self.workspace.device and t.dtype == dtype and tuple(t.shape) == tuple(shape) and t.is_contiguous()):
            raise ValueError(f"{what}: a contiguous {dtype} tensor of shape {tuple(shape)} on {self.workspace.device}")
        return t

    def _rows(self, hidden, weight, ids, teacher=None, temperature=1.0):
        c = self.cfg
        hs, ws = self._matrix(hidden, "hidden", self.hidden_dtype, c.dim), self._matrix(weight, "weight", self.weight_dtype, c.dim, c.vocab)
        n, entries = hidden.shape[0], 0
        if teacher is None:
            self._flat(ids, "targets", torch.int32, (n,))
        else:
            entries = ids.shape[1] if isinstance(ids, torch.Tensor) and ids.dim() == 2 else 0
            self._flat(ids, "ids", torch.int32, (n, entries))
            self._flat(teacher, "teacher", torch.float32, (n, entries))
        return tr_loss_rows(hidden.data_ptr(), weight.data_ptr(), hs, ws, ids.data_ptr(), None if teacher is None else teacher.data_ptr(), n, entries, float(temperature))

    def _out(self, t, what, n):
        return torch.empty(n, dtype=torch.float32, device=self.workspace.device) if t is None else self._flat(t, what, torch.float32, (n,))

    def _call(self, fn, what, *args):
        with torch.cuda.device(self.workspace.device):     # a default stream is the current device's
            rc = fn(C.byref(self.cfg), self.workspace.data_ptr(), self.workspace.numel(), self._stream(), *args)
        if rc:
            raise TokrouteError(rc, what)

    def _loss(self, fn, what, rows, loss, lse):
        loss, lse = self._out(loss, "loss", rows.rows), self._out(lse, "lse", rows.rows)
        self._call(fn, what, C.byref(rows), loss.data_ptr(), lse.data_ptr())
        return loss, lse

    def _grad(self, fn, what, rows, lse, grad_loss, d_hidden, d_weight):
        c, n, dev = self.cfg, rows.rows, self.workspace.device
        self._flat(lse, "lse", torch.float32, (n,))
        self._flat(grad_loss, "grad_loss", torch.float32, (n,))
        if d_hidden is None:
            d_hidden = torch.empty((n, c.dim), dtype=self.hidden_dtype, device=dev)
        if d_weight is None:
            d_weight = torch.empty((c.vocab, c.dim), dtype=self.weight_dtype, device=dev)
        out = tr_loss_grads(None, None, c.dim, c.dim)
        if d_hidden is not False:
            out.d_hidden_stride, out.d_hidden = self._matrix(d_hidden, "d_hidden", self.hidden_dtype, c.dim, n), d_hidden.data_ptr()
        if d_weight is not False:
            out.d_weight_stride, out.d_weight = self._matrix(d_weight, "d_weight", self.weight_dtype, c.dim, c.vocab), d_weight.data_ptr()
        self._call(fn, what, C.byref(rows), lse.data_ptr(), grad_loss.data_ptr(), C.byref(out))
        return (None if d_hidden is False else d_hidden), (None if d_weight is False else d_weight)

    # -- the ABI, same names
    def cross_entropy(self, hidden, weight, targets, loss=None, lse=None):
        """(loss, lse) of every row, float32 [n]: -log of the probability of targets[n] (device int32; below 0: the row does not count)."""
        return self._loss(self.lib.tr_cross_entropy, "tr_cross_entropy", self._rows(hidden, weight, targets), loss, lse)

    def cross_entropy_grad(self, hidden, weight, targets, lse, grad_loss, d_hidden=None, d_weight=None):
        """(d_hidden, d_weight): gradients of sum_n grad_loss[n] loss[n]. lse: as `cross_entropy` returned it on the same inputs. d_hidden and d_weight may be given
        (written over), or False: not computed."""
        return self._grad(self.lib.tr_cross_entropy_grad, "tr_cross_entropy_grad", self._rows(hidden, weight, targets), lse, grad_loss, d_hidden, d_weight)

    def distill(self, hidden, weight, ids, teacher, temperature=1.0, loss=None, lse=None):
        """(loss, lse) of every row: T^2 times the divergence from the teacher's distribution over its listed logits (ids device int32, teacher device float32,
        both [n][entries]; an id outside the vocabulary or a logit of -inf: no entry). lse is of the logits over T."""
        return self._loss(self.lib.tr_distill, "tr_distill", self._rows(hidden, weight, ids, teacher, temperature), loss, lse)

    def distill_grad(self, hidden, weight, ids, teacher, temperature, lse, grad_loss, d_hidden=None, d_weight=None):
        """(d_hidden, d_weight) of `distill`, like `cross_entropy_grad`."""
        return self._grad(self.lib.tr_distill_grad, "tr_distill_grad", self._rows(hidden, weight, ids, teacher, temperature), lse, grad_loss, d_hidden, d_weight)


class _CrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, plan, hidden, weight, targets):
        loss, lse = plan.cross_entropy(hidden, weight, targets)
        ctx.plan = plan
        ctx.save_for_backward(hidden, weight, targets, lse)
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_loss):
        hidden, weight, targets, lse = ctx.saved_tensors
        want = [None if need else False for need in ctx.needs_input_grad[1:3]]
        dh, dw = ctx.plan.cross_entropy_grad(hidden, weight, targets, lse, grad_loss.contiguous(), *want)
        return None, dh, dw, None


class _Distill(torch.autograd.Function):
    @staticmethod
    def forward(ctx, plan, hidden, weight, ids, teacher, temperature):
        loss, lse = plan.distill(hidden, weight, ids, teacher, temperature)
        ctx.plan, ctx.temperature = plan, temperature
        ctx.save_for_backward(hidden, weight, ids, teacher, lse)
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_loss):
        hidden, weight, ids, teacher, lse = ctx.saved_tensors
        want = [None if need else False for need in ctx.needs_input_grad[1:3]]
        dh, dw = ctx.plan.distill_grad(hidden, weight, ids, teacher, ctx.temperature, lse, grad_loss.contiguous(), *want)
        return None, dh, dw, None, None, None


def cross_entropy(plan: VocabLoss, hidden, weight, targets):
    """Per-row losses [n] of `VocabLoss.cross_entropy`, differentiable with respect to hidden and weight."""
    return _CrossEntropy.apply(plan, hidden, weight, targets)


def distill(plan: VocabLoss, hidden, weight, ids, teacher, temperature=1.0):
    """Per-row losses [n] of `VocabLoss.distill`, differentiable with respect to hidden and weight (the teacher is taken as given)."""
    return _Distill.apply(plan, hidden, weight, ids, teacher, float(temperature))
