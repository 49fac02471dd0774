"""The library's training operators as torch modules: a linear layer whose three products run in 8-bit
floating point (optionally with its neural gradient pruned first), an embedding whose gradient is summed
in a fixed order, and gradient clipping that stays on the device.

The modules marshal arguments for ``binding``; there is no CPU path.
"""
from __future__ import annotations

from typing import Dict, List, Optional, Sequence

import torch
from torch.autograd.function import once_differentiable

from . import binding as lgn


def _rows(t: torch.Tensor) -> torch.Tensor:
    """A matrix with contiguous rows that do not overlap: ``t`` as it is, or (transposed, broadcast) a copy."""
    if t.size(1) > 1 and t.stride(1) != 1 or t.size(0) > 1 and t.stride(0) < t.size(1):
        return t.contiguous()
    return t


def _pruned(dy: torch.Tensor, sparsity: float, seed: int, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Stochastic pruning of a neural gradient to the requested sparsity, threshold from its own statistics.  Entries that are
    not finite come out as NaN (the threshold is then without a meaning, and so are the others).  ``status``: int32
    word on the device that keeps the highest status seen."""
    g = dy.contiguous()
    if g.data_ptr() % 32 != 0:                                         # a contiguous slice, as the backward pass of torch.cat hands over
        g = g.clone()
    out = torch.empty_like(g)
    results, ws = lgn.new_results(1, g.device), lgn.new_workspace([g.numel()], g.device)
    with torch.cuda.device(g.device):                                  # the grouped call takes the current device's stream
        lgn.lgn_compress_layers([lgn.make_layer(g, out, lgn.MODE_PRUNE, S=sparsity, seed=seed)], results, ws)
    out.add_(g, alpha=0.0)                                             # adds 0, or NaN: pruning is for finite values and may drop others
    if status is not None:
        torch.maximum(status, lgn.status_of(results), out=status)
    return out


class _LinearFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, sparsity, seed, status):
        wq, wqt = lgn.lgn_fp8_quantize(_rows(weight), lgn.E4M3, lgn.BLOCK_SQUARE, transposed=True)
        xq, xqt = lgn.lgn_fp8_quantize(_rows(x), lgn.E4M3, transposed=True)
        ctx.save_for_backward(wqt._buffer, xqt._buffer)
        ctx.extents = [(q.rows, q.k, q.fmt) for q in (wqt, xqt)]
        ctx.sparsity, ctx.seed, ctx.status, ctx.dtypes = sparsity, seed, status, (x.dtype, weight.dtype)
        return lgn.lgn_fp8_matmul(xq, wq, out_dtype=x.dtype, status=status)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        need_dx, need_dw = ctx.needs_input_grad[:2]
        if not (need_dx or need_dw):
            return None, None, None, None, None
        wqt, xqt = (lgn.Fp8Operand._of_buffer(t, *e) for t, e in zip(ctx.saved_tensors, ctx.extents))
        if ctx.sparsity > 0.0:
            dy = _pruned(dy, ctx.sparsity, ctx.seed, ctx.status)
        dq, dqt = lgn.lgn_fp8_quantize(_rows(dy), lgn.E5M2, rowwise=need_dx, transposed=need_dw)
        dx = lgn.lgn_fp8_matmul(dq, wqt, out_dtype=ctx.dtypes[0], status=ctx.status) if need_dx else None
        dw = lgn.lgn_fp8_matmul(dqt, xqt, out_dtype=ctx.dtypes[1], status=ctx.status) if need_dw else None
        return dx, dw, None, None, None


class Fp8Linear(torch.nn.Module):
    """y = x W^T with x, W and the incoming gradient in 8-bit floating point (E4M3, E4M3, E5M2; one power-of-two
    scale per block of 128), fp32 sums.  ``sparsity`` > 0 prunes the incoming gradient to that fraction of zeros
    before the two backward products, with random numbers that depend on ``seed`` and the place alone: it changes from step to step
    (advance() adds 1), and layers want seeds that do not meet (the example takes multiples of 2^32).  Pruning is for
    magnitudes below 2^104; entries that are not finite come through as NaN, as they do without pruning.  The waits on the
    device are bounded; check() tells whether one ran out."""

    def __init__(self, in_features: int, out_features: int, sparsity: float = 0.0, device=None, seed: int = 0):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.empty(out_features, in_features, device=device))
        torch.nn.init.normal_(self.weight, std=in_features ** -0.5)
        self.sparsity, self.seed = float(sparsity), int(seed)
        self._status: Dict[torch.device, torch.Tensor] = {}            # an int32 word on each device a pass has run on

    def advance(self) -> None:
        self.seed += 1

    def check(self) -> None:
        """Raises LgnError (LGN_ERR_TIMEOUT) if a device-side wait of the passes since the last check ran out: what they
        computed is then not valid.  Waits for the device."""
        codes = []
        for device, word in self._status.items():
            torch.cuda.synchronize(device)                             # passes on any of its streams
            codes.append(int(word.item()))
            word.zero_()
        if any(codes):
            raise lgn.LgnError(max(codes), "Fp8Linear")

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        if x.device not in self._status:
            self._status[x.device] = torch.zeros(1, dtype=torch.int32, device=x.device)
        y = _LinearFn.apply(x.reshape(-1, x.shape[-1]), self.weight, self.sparsity, self.seed, self._status[x.device])
        return y.reshape(*x.shape[:-1], self.weight.shape[0])


class _EmbeddingFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, weight, ids, scale, padding_idx, out_dtype):
        ctx.save_for_backward(ids)
        ctx.args = (weight.shape[0], scale, padding_idx, weight.dtype)
        return lgn.lgn_embedding(_rows(weight), ids, scale, out_dtype=out_dtype)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        (ids,) = ctx.saved_tensors
        vocab, scale, padding_idx, dtype = ctx.args
        return lgn.lgn_embedding_grad(_rows(dout), ids, vocab, scale, padding_idx, out_dtype=dtype), None, None, None, None


class Embedding(torch.nn.Module):
    """scale * weight[ids]; ids outside the table give zeros.  The gradient leaves padding_idx out."""

    def __init__(self, vocab: int, dim: int, scale: float = 1.0, padding_idx: int = -1,
                 out_dtype: torch.dtype = torch.bfloat16, device=None):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.empty(vocab, dim, device=device))
        torch.nn.init.normal_(self.weight, std=1.0 / scale)
        self.scale, self.padding_idx, self.out_dtype = float(scale), int(padding_idx), out_dtype

    def forward(self, ids: torch.Tensor) -> torch.Tensor:
        flat = ids.reshape(-1).contiguous()
        out = _EmbeddingFn.apply(self.weight, flat, self.scale, self.padding_idx, self.out_dtype)
        return out.reshape(*ids.shape, self.weight.shape[1])


class GradClipper:
    """Clips the gradients of a fixed list of parameters by their global norm, in place, without a host round
    trip.  A gradient has to stay where it is from the first clip() that finds it (zero_grad(set_to_none=False)); a
    parameter without one yet takes part from the step that brings it."""

    def __init__(self, parameters: Sequence[torch.nn.Parameter], max_norm: float):
        self._params, self.max_norm = list(parameters), float(max_norm)
        self._grads: List[Optional[torch.Tensor]] = [None] * len(self._params)
        self._take()
        if self._list.count == 0:
            raise ValueError("no parameter has a gradient yet")
        self._device = next(g for g in self._grads if g is not None).device
        self.record = lgn.new_norm_record(self._device)
        self._ws = lgn.new_clip_workspace(self._device, len(self._params))

    def _take(self) -> None:
        """Descriptors of the gradients that there are."""
        self._grads = [p.grad for p in self._params]
        self._list = lgn.make_grads([g for g in self._grads if g is not None])
        self._places = [None if g is None else g.data_ptr() for g in self._grads]

    def clip(self, stream=None) -> torch.Tensor:
        """Scales the gradients; returns their norm before it, a scalar on the device that later calls leave alone.  It is part
        of the call's record, which is ``record`` until the next call."""
        more = False
        for p, g, at in zip(self._params, self._grads, self._places):
            if g is None:
                more = more or p.grad is not None
            elif p.grad is not g or g.data_ptr() != at:
                raise RuntimeError("a gradient has been replaced since the clipper was made")
        if more:
            self._take()
        if stream is not None and not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(int(stream), self._device)
        self.record = lgn._empty(self.record.shape, torch.uint8, self._device, stream)
        lgn.lgn_clip_grad_norm(self._list, self.max_norm, self.record, self._ws, stream)
        return lgn.norm_of(self.record)
