"""Tokens drawn from rows of logits, and a row's largest logits.

The binding of tr_sample and tr_top (include/tokroute.h states what they compute, and what becomes of infinities, NaN and rows without any token). A `Sampler` keeps the workspace
that calls share; `Draw` is how `joint.generate` draws. There is no CPU fallback: without the built library or without a GPU calls raise.
"""
from __future__ import annotations

import ctypes as C
import operator
from dataclasses import dataclass

import torch
from torch.autograd.graph import increment_version

from . import tokroute
from .tokroute import TokrouteError, tr_pick_config, tr_pick_rows, tr_sample_how

MOST_ENTRIES, MOST_VOCAB = 1024, 1 << 20     # that tr_top lists, and that the calls take

_DTYPES = {torch.float32: tokroute.F32, torch.bfloat16: tokroute.BF16}


def _int32(v):
    """A number beyond 32 bits as the nearest that has them, which the library judges (ctypes would take its last 32 bits)."""
    return max(min(operator.index(v), 2**31 - 1), -2**31)


@dataclass(frozen=True)
class Draw:
    """How tokens are drawn: the arguments of `Sampler.sample` of the same names. temperature 0: the largest logit."""
    temperature: float = 1.0
    top_k: int = 0
    top_p: float = 1.0
    min_p: float = 0.0


class Sampler:
    """Workspace and sizes of calls on up to max_rows rows of `vocab` logits.

    Calls enqueue on the current stream of `device`, whichever device is current; calls of one Sampler on different streams must be ordered by the caller, since they share the workspace.
    Rows may be strided; each row is contiguous.
    """

    def __init__(self, max_rows: int, vocab: int, dtype=torch.float32, device="cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("tokroute needs a GPU: no CPU path exists")
        if dtype not in _DTYPES:
            raise ValueError(f"logits are float32 or bfloat16, not {dtype}")
        self.lib = tokroute.load_library()
        self.dtype = dtype
        self.cfg = tr_pick_config(_int32(max_rows), _int32(vocab), _DTYPES[dtype])
        nbytes = self.lib.tr_pick_workspace_bytes(C.byref(self.cfg))
        if nbytes == 0:
            raise TokrouteError(tokroute.ERR_SHAPE, "tr_pick_workspace_bytes", "(sizes or types not supported)")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.device = self.workspace.device
        self._home = torch.cuda.current_stream(self.device).cuda_stream

    # -- helpers
    def _rows(self, logits):
        v = self.cfg.vocab
        fine = isinstance(logits, torch.Tensor) and logits.dtype == self.dtype and logits.device == self.device and logits.dim() == 2
        (n, columns), (stride, along) = (logits.shape, logits.stride()) if fine else ((0, 0), (0, 0))
        if columns != v or (along != 1 and v > 1):
            raise ValueError(f"logits: a {self.dtype} matrix of {v} columns with contiguous rows on {self.device}")
        return tr_pick_rows(logits.data_ptr(), max(stride, v) if n <= 1 else stride, n if n < 2**31 else 2**31 - 1)      # (more than any Sampler is for)

    def _flat(self, t, what, dtype, shape):
        if not (isinstance(t, torch.Tensor) and t.dtype == dtype and t.device == self.device and t.shape == shape and t.is_contiguous()):
            raise ValueError(f"{what}: a contiguous {dtype} tensor of shape {shape} on {self.device}")
        return t.data_ptr()

    def _over(self, t, what, dtype, shape):
        self._flat(t, what, dtype, shape)
        increment_version(t)      # autograd sees what is written over

    def _call(self, fn, what, *args):
        stream = tokroute.raw_stream(self.device.index)
        if stream != self._home:
            self.workspace.record_stream(torch.cuda.current_stream(self.device))    # its memory is not handed on while work of that stream may use it
        with tokroute.on_device(self.device.index):      # a default stream is the current device's
            rc = fn(C.byref(self.cfg), self.workspace.data_ptr(), self.workspace.numel(), stream, *args)
        if rc:
            raise TokrouteError(rc, what)

    # -- the ABI, same names
    def sample(self, logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, token=None, logprob=None):
        """(token int32 [n], logprob float32 [n]): one token a row from its random number u (float32 [n] in [0, 1)), and the logarithm of its probability among what the filters keep.

        temperature, top_p, min_p (float32 [n]) and top_k (int32 [n]) are numbers or device tensors with a value a row. token and logprob may be given (written over)."""
        rows = self._rows(logits)
        shape = (rows.rows,)
        how = tr_sample_how(self._flat(u, "u", torch.float32, shape))
        if isinstance(temperature, torch.Tensor):
            how.temperatures = self._flat(temperature, "temperature", torch.float32, shape)
        else:
            how.temperature = temperature
        if isinstance(top_k, torch.Tensor):
            how.top_ks = self._flat(top_k, "top_k", torch.int32, shape)
        else:
            how.top_k = _int32(top_k)
        if isinstance(top_p, torch.Tensor):
            how.top_ps = self._flat(top_p, "top_p", torch.float32, shape)
        else:
            how.top_p = top_p
        if isinstance(min_p, torch.Tensor):
            how.min_ps = self._flat(min_p, "min_p", torch.float32, shape)
        else:
            how.min_p = min_p
        if token is None:
            token = torch.empty_like(u, dtype=torch.int32)
        else:
            self._over(token, "token", torch.int32, shape)
        if logprob is None:
            logprob = torch.empty_like(u)
        else:
            self._over(logprob, "logprob", torch.float32, shape)
        self._call(self.lib.tr_sample, "tr_sample", C.byref(rows), C.byref(how), token.data_ptr(), logprob.data_ptr())
        return token, logprob

    def top(self, logits, entries: int, ids=None, values=None):
        """(ids int32 [n][entries], values float32 [n][entries]): the largest logits of each row, in falling order, equal ones by id; -1 and -inf where a row has fewer."""
        if entries > MOST_ENTRIES:
            raise TokrouteError(tokroute.ERR_CAPACITY, "tr_top", f"(more than {MOST_ENTRIES} entries)")
        rows = self._rows(logits)
        shape = (rows.rows, entries)
        if ids is None:
            ids = logits.new_empty(shape, dtype=torch.int32)
        else:
            self._over(ids, "ids", torch.int32, shape)
        if values is None:
            values = logits.new_empty(shape, dtype=torch.float32)
        else:
            self._over(values, "values", torch.float32, shape)
        self._call(self.lib.tr_top, "tr_top", C.byref(rows), entries, ids.data_ptr(), values.data_ptr())
        return ids, values
