"""The length of many gradients together, and its clipping: the binding of tr_grad_norm and tr_grad_clip (include/tokroute.h).

There is no CPU fallback: without the built library or without a GPU calls raise.
"""
from __future__ import annotations

from array import array

import torch
from torch.autograd.graph import increment_version

from . import tokroute
from .tokroute import TokrouteError

_type_of = torch.Tensor.dtype.__get__
_DTYPES = {torch.float32: tokroute.F32, torch.bfloat16: tokroute.BF16}


def _dense(t):
    """Whether a tensor's elements fill one piece of memory, in whatever order of its dimensions."""
    return t.is_contiguous() or t.permute(sorted(range(t.dim()), key=lambda i: (-t.stride(i), -t.shape[i]))).is_contiguous()


class Clipper:
    """Workspace of the calls. Calls enqueue on the current stream of `device`, whichever device is current; calls of one Clipper on different streams must be ordered by the caller.

    Gradients are float32 or bfloat16 tensors on `device`, of any mixture of sizes, each of elements that fill one piece of memory; None (a parameter without a gradient) is left out.
    """

    def __init__(self, device="cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("tokroute needs a GPU: no CPU path exists")
        self.lib = tokroute.load_library()
        self.workspace = torch.empty(self.lib.tr_grad_workspace_bytes(), dtype=torch.uint8, device=device)
        self.device = self.workspace.device
        self._home = torch.cuda.current_stream(self.device).cuda_stream

    # -- helpers
    def _look(self, grads, what="gradients"):
        """Addresses, the types there are, and whether all are contiguous; a few calls over all tensors rather than several a tensor (hundreds of gradients take longer to look at than to read)."""
        try:
            kinds = set(map(_type_of, grads))
            fine = kinds <= _DTYPES.keys() and set(map(torch.Tensor.get_device, grads)) <= {self.device.index} and all(map(torch.Tensor.is_contiguous, grads))
        except (TypeError, RuntimeError):       # no tensor, or one of another layout
            fine = False
        if not fine and not all(isinstance(t, torch.Tensor) and t.dtype in _DTYPES and t.device == self.device and t.layout == torch.strided and _dense(t) for t in grads):
            raise ValueError(f"{what}: float32 or bfloat16 tensors on {self.device}, each of elements that fill one piece of memory")
        return array("q", list(map(torch.Tensor.data_ptr, grads))), kinds, fine

    @staticmethod
    def _sizes(grads, kinds, counts):
        types = [_DTYPES[kind] for kind in kinds] * len(grads) if len(kinds) == 1 else [_DTYPES[t.dtype] for t in grads]
        return array("q", counts), array("i", types)

    def _call(self, fn, what, arrays, *args):
        stream = tokroute.raw_stream(self.device.index)
        if stream != self._home:
            self.workspace.record_stream(torch.cuda.current_stream(self.device))    # its memory is not handed on while work of that stream may use it
        with tokroute.on_device(self.device.index):      # a default stream is the current device's
            rc = fn(self.workspace.data_ptr(), self.workspace.numel(), stream, len(arrays[0]), *[x.buffer_info()[0] for x in arrays], *args)
        if rc:
            raise TokrouteError(rc, what)

    # -- the ABI
    def norm(self, grads):
        """Length of all gradients together: a float32 tensor of no dimensions."""
        grads = [t for t in grads if t is not None]
        (at, kinds, _), norm = self._look(grads), torch.empty((), dtype=torch.float32, device=self.device)
        self._call(self.lib.tr_grad_norm, "tr_grad_norm", [at, *self._sizes(grads, kinds, list(map(torch.Tensor.numel, grads)))], norm.data_ptr())
        return norm

    def clip(self, grads, max_norm: float, out=None):
        """The same, and the gradients scaled by min(1, max_norm / norm): in place, or into `out` (tensors of the same types, shapes and strides, None where a gradient is None;
        where all are contiguous those of as many elements will do)."""
        all_grads = list(grads)
        all_out = all_grads if out is None else list(out)
        grads, out = [t for t in all_grads if t is not None], [t for t in all_out if t is not None]
        if len(all_out) != len(all_grads) or len(out) != len(grads) or (len(grads) < len(all_grads) and any((a is None) != (b is None) for a, b in zip(all_grads, all_out))):
            raise ValueError("out: a tensor for every gradient")
        at, kinds, plain = self._look(grads)
        to, counts = at, list(map(torch.Tensor.numel, grads))
        if any(a is not b for a, b in zip(grads, out)):
            to, out_kinds, out_plain = self._look(out, "out")
            alike = kinds == out_kinds and (len(kinds) <= 1 or list(map(_type_of, grads)) == list(map(_type_of, out)))
            if plain and out_plain:
                alike = alike and counts == list(map(torch.Tensor.numel, out))
            else:
                alike = alike and all(a.shape == b.shape and (a.stride() == b.stride() or (a.is_contiguous() and b.is_contiguous())) for a, b in zip(grads, out))
            if not alike:
                raise ValueError("out: tensors of the gradients' types, shapes and strides")
        norm = torch.empty((), dtype=torch.float32, device=self.device)
        self._call(self.lib.tr_grad_clip, "tr_grad_clip", [at, to, *self._sizes(grads, kinds, counts)], max_norm, norm.data_ptr())
        increment_version(out)      # autograd sees what is written over
        return norm
