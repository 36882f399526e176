"""The optimizer of the dense side: what a training loop calls between the dense model's backward
pass and the next batch, beside the tables' own update (ss_embbag_backward_update).

    opt = AdamW(params, lr=1e-3, max_norm=1.0, state_bits=8, master=True)
    opt.set_grads([p.grad for p in params])
    opt.step()

This class only owns buffers and issues the library calls in order; nothing in set_grads, step and
moments synchronises with the host.  step() can be captured in a graph: steps are counted on the
device, and with lr a device tensor the schedule is, too.
"""
from __future__ import annotations

from typing import Optional, Sequence

import torch

from . import binding as B


class AdamW:
    """AdamW over all of `params` in one launch (fp32, bf16 and fp16 mixed as they come).

    state_bits  32, or 8: packed moments, 2 bytes per element instead of 8
    master      keep fp32 copies of the 16-bit parameters
    no_decay    truth values, one per tensor: weight decay leaves those out
    max_norm    clip the gradients' common norm, and leave a step out where it is not finite
    grad_scale  what the gradients are multiplied by first (the inverse of a loss scale); used
                with max_norm (float("inf"): scale and check, do not clip)
    """

    def __init__(self, params: Sequence[torch.Tensor], lr=1e-3, betas=(0.9, 0.999),
                 eps: float = 1e-8, weight_decay: float = 0.01, state_bits: int = 32,
                 master: bool = False, no_decay: Optional[Sequence[bool]] = None,
                 grad_dtypes: Optional[Sequence[torch.dtype]] = None,
                 max_norm: Optional[float] = None, grad_scale: float = 1.0):
        params = [p.detach() for p in params]
        if grad_dtypes is None:
            grad_dtypes = [p.dtype for p in params]
        self.list = B.TensorList(params, grad_dtypes=grad_dtypes, no_decay=no_decay)
        self.state = B.AdamWState(self.list, state_bits, master)
        self.lr, self.betas, self.eps = lr, betas, eps
        self.weight_decay, self.max_norm, self.grad_scale = weight_decay, max_norm, grad_scale
        self.clip: Optional[torch.Tensor] = None
        if max_norm is not None:
            dev = self.list.device
            self.clip = torch.zeros(4, device=dev)
            self._ws = torch.empty(B.ss_grad_norm_workspace_bytes(self.list), dtype=torch.uint8,
                                   device=dev)
        elif grad_scale != 1.0:
            raise B.SlipstreamError("AdamW: grad_scale needs max_norm (float('inf') to not clip)")

    def set_grads(self, grads: Sequence[torch.Tensor], stream=None) -> None:
        """The gradient tensors that steps read from now on."""
        self.list.set_grads(grads, stream)

    def set_step(self, steps: int, stream=None) -> None:
        """Number of steps taken so far (a restored state's).  With a stream the count is set in order
        on it, and under capture on the current one; otherwise the call waits for the device on
        both sides, so that it comes behind the steps of every stream and before those that
        follow."""
        if steps < 0:
            raise B.SlipstreamError(f"set_step: steps = {steps}")
        count = self.state.counters[:1]
        if stream is not None:
            with torch.cuda.stream(stream):
                count.fill_(steps)
        elif torch.cuda.is_current_stream_capturing():
            count.fill_(steps)
        else:
            torch.cuda.synchronize(self.list.device)
            count.fill_(steps)
            torch.cuda.synchronize(self.list.device)

    def steps(self, stream=None) -> int:
        """Steps taken so far; waits for the device (while no stream of it is under capture), with a
        stream for that one only."""
        return self._counter(0, stream)

    def left_out(self, stream=None) -> int:
        """Steps left out because the gradients' norm was not finite; waits as steps()."""
        return self._counter(1, stream)

    def _counter(self, k: int, stream) -> int:
        # (reading a tensor waits for the current stream alone; steps may run on others)
        if stream is None:
            torch.cuda.synchronize(self.list.device)
            return int(self.state.counters[k])
        with torch.cuda.stream(stream):
            return int(self.state.counters[k])

    def step(self, clip: Optional[torch.Tensor] = None, stream=None) -> None:
        """clip: fp32 [4] as ss_grad_norm writes it (one norm over several optimizers, say); without
        it and with max_norm the norm of this optimizer's gradients is taken first."""
        if clip is None and self.max_norm is not None:
            B.ss_grad_norm(self.list, self.max_norm, self.clip, self._ws, self.grad_scale, stream)
            clip = self.clip
        B.ss_adamw_step(self.list, self.state, self.lr, self.betas[0], self.betas[1], self.eps,
                        self.weight_decay, clip, stream)

    def moments(self, m: torch.Tensor, v: torch.Tensor, stream=None) -> None:
        """The values of 8-bit moments, as bf16 [state_elems]."""
        B.ss_adamw_moments(self.list, self.state, m, v, stream)
