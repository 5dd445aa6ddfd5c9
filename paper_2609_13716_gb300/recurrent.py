"""The gated linear recurrence and the orthogonalised update for torch programs: an autograd
function over the sequence, a serving step and an optimiser, all through the C ABI
(aht_glr_forward / aht_glr_backward / aht_muon_step); no step of their arithmetic is torch's.
"""
from __future__ import annotations

import contextlib

import torch

from . import aht


_here = contextlib.nullcontext()


def _device_of(t):
    """The device of a CUDA tensor made the current one (other tensors are refused where they are used)."""
    return torch.cuda.device(t.device) if t.is_cuda and t.get_device() != torch.cuda.current_device() else _here


def _written(t):
    """Tells autograd that the library wrote a tensor in place, as torch's own in-place operations do: a
    graph that saved its earlier value raises instead of using the new one."""
    if not t.is_inference():
        torch.autograd.graph.increment_version(t)


class _GatedRecurrence(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, r, i, lam, h0, reset, lengths):
        T, N, D = x.shape
        h = torch.empty(T, N, D, dtype=x.dtype, device=x.device)
        h_last = torch.empty(N, D, dtype=torch.float32, device=x.device)
        need = any(ctx.needs_input_grad)
        ckpt = torch.empty(aht.aht_glr_ckpt_shape(T, N, D), device=x.device) if need else None
        with _device_of(x):
            aht.aht_glr_forward(x, r, i, lam, h, reset=reset, lengths=lengths, h0=h0, h_last=h_last, ckpt=ckpt)
        if need:
            ctx.save_for_backward(x, r, i, lam, ckpt, reset, lengths)
        return h, h_last

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dh, dh_last):
        x, r, i, lam, ckpt, reset, lengths = ctx.saved_tensors
        T, N, D = x.shape
        # the three gradients side by side, one allocation (autograd still concatenates them into a new
        # tensor where x, r and i are slices of one projection)
        grad = torch.empty(T, N, 3 * D, dtype=x.dtype, device=x.device)
        dx, dr, di = grad.split(D, dim=2)
        dlam = torch.empty(D, device=x.device)
        dh0 = torch.empty(N, D, device=x.device) if ctx.needs_input_grad[4] else None
        ws = torch.empty(aht.aht_glr_workspace(T, N, D), dtype=torch.uint8, device=x.device)
        if dh is not None and dh.stride(2) != 1:
            dh = dh.contiguous()
        with _device_of(x):
            aht.aht_glr_backward(x, r, i, lam, ckpt, dh, dx, dr, di, dlam, ws, reset=reset, lengths=lengths,
                                 dh_last=None if dh_last is None else dh_last.contiguous(), dh0=dh0)
        return dx, dr, di, dlam, dh0, None, None


def gated_recurrence(x, r, i, lam, h0=None, reset=None, lengths=None):
    """h [T][N][D] and the final state f32 [N][D] of the recurrence over x, r, i [T][N][D]
    (f32 or bf16; any step and env strides), differentiable in x, r, i, lam and h0."""
    return _GatedRecurrence.apply(x, r, i, lam, h0, reset, lengths)


@torch.no_grad()
def gated_step(x, r, i, lam, state, reset=None):
    """One serving step over x, r, i [N][D]: updates ``state`` (f32 [N][D]) in place and
    returns h [N][D]."""
    h = torch.empty(1, *x.shape, dtype=x.dtype, device=x.device)
    with _device_of(x):
        aht.aht_glr_forward(x[None], r[None], i[None], lam, h, reset=None if reset is None else reset[None], h0=state,
                            h_last=state)
    _written(state)
    return h[0]


class OrthogonalOptimizer:
    """aht_muon_step over the gradients of a fixed list of f32 matrices.  The updates run on the
    stream that is current here; a step under another one is ordered with it both ways.

    step() needs a gradient of every matrix and clears it.  What there is to save and load beside
    the parameters is ``momenta``, a list of tensors in their order."""

    def __init__(self, params, lr=0.02, **cfg):
        self.params, self.lr = list(params), lr
        self.momenta = [torch.zeros_like(p) for p in self.params]
        device = self.params[0].device if self.params else None
        self.stream = torch.cuda.current_stream(device)
        with torch.cuda.device(device):
            self.handle = aht.aht_muon_create([tuple(p.shape) for p in self.params], stream=self.stream, **cfg)

    @torch.no_grad()
    def step(self):
        now = torch.cuda.current_stream(self.stream.device)
        if now != self.stream:
            self.stream.wait_stream(now)
        aht.aht_muon_step(self.handle, [p.detach() for p in self.params], self.momenta, [p.grad for p in self.params],
                          self.lr)
        if now != self.stream:
            now.wait_stream(self.stream)
        for p in self.params:
            _written(p)
            p.grad.record_stream(self.stream)  # wherever it was allocated: its memory is not used again before
            p.grad = None

    def sync(self):
        """Waits for the updates and raises what the device reported."""
        aht.aht_muon_sync(self.handle)
