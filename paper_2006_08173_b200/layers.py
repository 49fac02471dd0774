"""The library's training operators as torch modules: a linear layer whose three products run in 8-bit
floating point (optionally with its neural gradient pruned first), one whose forward product runs in 8-bit integers, linear
layers of experts over rows grouped by expert, an embedding whose gradient is summed in a fixed order, the loss against a
teacher's top logits, and gradient clipping that stays on the device.

The modules marshal arguments for ``binding``; there is no CPU path.  A step may be captured into a CUDA graph after a pass on the same
device (which makes the status words), and while no graph of autograd from outside of the capture holds the same parameters:
torch would have the captured gradients wait for its stream.
"""
from __future__ import annotations

from typing import Dict, List, Optional, Sequence, Tuple

import torch
from torch.autograd.forward_ad import unpack_dual
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


class _Bounded(torch.nn.Module):
    """A module whose kernels' waits are bounded: an int32 word on each device a pass has run on keeps the highest status."""

    def __init__(self):
        super().__init__()
        self._status: Dict[torch.device, torch.Tensor] = {}

    def _status_on(self, device: torch.device) -> torch.Tensor:
        if device not in self._status:
            if device.type != "cuda":                                  # check() would wait for it
                raise ValueError("the module computes on CUDA tensors")
            with torch.inference_mode(False):                          # check() writes it outside of that mode too
                self._status[device] = torch.zeros(1, dtype=torch.int32, device=device)
        return self._status[device]

    def check(self) -> None:
        """Raises LgnError (LGN_ERR_TIMEOUT) if a device-side wait of the passes since the last check ran out: what they
        computed is then not valid.  Waits for the device."""
        codes = []
        for device, word in self._status.items():
            torch.cuda.synchronize(device)                             # passes on any of its streams
            codes.append(int(word.item()))
            word.zero_()
        if any(codes):
            raise lgn.LgnError(max(codes), type(self).__name__)


class Fp8Linear(_Bounded):
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

    def advance(self) -> None:
        self.seed += 1

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        y = _LinearFn.apply(x.reshape(-1, x.shape[-1]), self.weight, self.sparsity, self.seed, self._status_on(x.device))
        return y.reshape(*x.shape[:-1], self.weight.shape[0])


class _Int8LinearFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, sparsity, seed, status):
        need_dx, need_dw = ctx.needs_input_grad[:2]
        wqt = lgn.lgn_fp8_quantize(_rows(weight), lgn.E4M3, lgn.BLOCK_SQUARE, rowwise=False, transposed=True)[1] if need_dx else None
        xqt = lgn.lgn_fp8_quantize(_rows(x), lgn.E4M3, rowwise=False, transposed=True)[1] if need_dw else None
        kept = [q for q in (wqt, xqt) if q is not None]
        ctx.save_for_backward(*(q._buffer for q in kept))
        ctx.extents = [(q.rows, q.k, q.fmt) for q in kept]
        ctx.sparsity, ctx.seed, ctx.status, ctx.dtypes = sparsity, seed, status, (x.dtype, weight.dtype)
        return lgn.lgn_int8_matmul(lgn.lgn_int8_quantize(_rows(x)), lgn.lgn_int8_quantize(_rows(weight)), out_dtype=x.dtype, status=status)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        need_dx, need_dw = ctx.needs_input_grad[:2]
        if not (need_dx or need_dw):
            return None, None, None, None, None
        kept = [lgn.Fp8Operand._of_buffer(t, *e) for t, e in zip(ctx.saved_tensors, ctx.extents)]
        if ctx.sparsity > 0.0:
            dy = _pruned(dy, ctx.sparsity, ctx.seed, ctx.status)
        dq, dqt = lgn.lgn_fp8_quantize(_rows(dy), lgn.E5M2, rowwise=need_dx, transposed=need_dw)
        dx = lgn.lgn_fp8_matmul(dq, kept[0], out_dtype=ctx.dtypes[0], status=ctx.status) if need_dx else None
        dw = lgn.lgn_fp8_matmul(dqt, kept[-1], out_dtype=ctx.dtypes[1], status=ctx.status) if need_dw else None
        return dx, dw, None, None, None


class Int8Linear(_Bounded):
    """y = x W^T with x and W in 8-bit integers, one scale per row of either, for a layer that is to serve that way.  Its gradients are taken as if
    nothing had been rounded, in the 8-bit floating point of Fp8Linear: neural gradients span more binades than 8-bit integers have.
    ``sparsity``, ``seed``, advance() and check() are as there.  freeze() lays the weights out once for passes without gradients."""

    def __init__(self, in_features: int, out_features: int, sparsity: float = 0.0, device=None, seed: int = 0):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.empty(out_features, in_features, device=device))
        torch.nn.init.normal_(self.weight, std=in_features ** -0.5)
        self.sparsity, self.seed = float(sparsity), int(seed)
        self._frozen: Optional[lgn.Int8Operand] = None

    def advance(self) -> None:
        self.seed += 1

    def freeze(self, frozen: bool = True) -> None:
        """From here on the layer computes with the weights as they are now, and refuses passes that want derivatives, in either mode; ``frozen`` false: as
        before."""
        self._frozen = lgn.lgn_int8_quantize(_rows(self.weight.detach())) if frozen else None

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        flat, status = x.reshape(-1, x.shape[-1]), self._status_on(x.device)
        if self._frozen is None:
            y = _Int8LinearFn.apply(flat, self.weight, self.sparsity, self.seed, status)
        elif torch.is_grad_enabled() and (x.requires_grad or self.weight.requires_grad):
            raise RuntimeError("the layer is frozen: no gradients")
        elif unpack_dual(x).tangent is not None or unpack_dual(self.weight).tangent is not None:
            raise RuntimeError("the layer is frozen: no tangents")
        else:
            y = lgn.lgn_int8_matmul(lgn.lgn_int8_quantize(_rows(flat)), self._frozen, out_dtype=x.dtype, status=status)
        return y.reshape(*x.shape[:-1], self.weight.shape[0])


def by_expert(ids: torch.Tensor, experts: int) -> Tuple[torch.Tensor, torch.Tensor]:
    """(order, offsets) of a flat tensor of expert numbers: ids[order] is sorted, equal ones in the order they came, and expert e has the places
    offsets[e] to offsets[e + 1] of it.  Numbers outside [0, experts) come ahead of or behind all of them.  Nothing leaves the device."""
    if ids.dtype not in (torch.int32, torch.int64):
        ids = ids.long()                                               # narrow ones do not hold the number of experts
    ranked, order = torch.sort(ids, stable=True)
    return order, torch.searchsorted(ranked, torch.arange(experts + 1, dtype=ids.dtype, device=ids.device))


class _ExpertFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, offsets, sparsity, seed, status):
        xb, wb = x.to(torch.bfloat16), weight.to(torch.bfloat16)
        need_dx, need_dw = ctx.needs_input_grad[:2]
        ctx.save_for_backward(offsets, *([wb] if need_dx else []), *([xb] if need_dw else []))
        ctx.sparsity, ctx.seed, ctx.status, ctx.dtypes = sparsity, seed, status, (x.dtype, weight.dtype)
        return lgn.lgn_grouped_matmul(xb, wb, offsets, out_dtype=x.dtype, status=status)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        need_dx, need_dw = ctx.needs_input_grad[:2]
        if not (need_dx or need_dw):
            return None, None, None, None, None, None
        offsets, *kept = ctx.saved_tensors
        if ctx.sparsity > 0.0:                                         # whatever stands in rows of no expert must not reach the threshold
            row = torch.arange(dy.shape[0], device=dy.device)
            dy = dy.masked_fill(((row < offsets[0]) | (row >= offsets.max()))[:, None], 0.0)
            dy = _pruned(dy, ctx.sparsity, ctx.seed, ctx.status)
        dy = dy.to(torch.bfloat16)
        dx = lgn.lgn_grouped_matmul(dy, kept[0], offsets, out_dtype=ctx.dtypes[0], transposed=True, status=ctx.status) if need_dx else None
        dw = lgn.lgn_grouped_weight_grad(dy, kept[-1], offsets, out_dtype=ctx.dtypes[1], status=ctx.status) if need_dw else None
        return dx, dw, None, None, None, None


class ExpertLinear(_Bounded):
    """y[r] = W_e x[r] for the rows r = offsets[e] .. offsets[e + 1] - 1 of each expert e (by_expert gives such offsets), in bf16 with fp32 sums; rows of no
    expert give zeros.  ``sparsity``, ``seed``, advance() and check() are those of Fp8Linear; rows of no expert count as zeros there."""

    def __init__(self, experts: int, in_features: int, out_features: int, sparsity: float = 0.0, device=None, seed: int = 0):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.empty(experts, out_features, in_features, device=device))
        torch.nn.init.normal_(self.weight, std=in_features ** -0.5)
        self.sparsity, self.seed = float(sparsity), int(seed)

    def advance(self) -> None:
        self.seed += 1

    def forward(self, x: torch.Tensor, offsets: torch.Tensor) -> torch.Tensor:
        return _ExpertFn.apply(x, self.weight, offsets, self.sparsity, self.seed, self._status_on(x.device))


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


class _DistillFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, ids, teacher, labels, temperature, alpha):
        ctx.save_for_backward(logits, ids, teacher, labels)
        ctx.args = (temperature, alpha)
        return lgn.lgn_distill_loss(_rows(logits), ids, teacher, labels, temperature, alpha)[0]

    @staticmethod
    @once_differentiable
    def backward(ctx, dloss):
        logits, ids, teacher, labels = ctx.saved_tensors
        temperature, alpha = ctx.args
        dlogits = lgn.lgn_distill_loss(_rows(logits), ids, teacher, labels, temperature, alpha, dloss.float().contiguous(), grad=True)[1]
        return dlogits, None, None, None, None, None


class DistillLoss(torch.nn.Module):
    """Losses of rows of logits against a teacher's logits at its top places: alpha T^2 times the divergence of the student's softmax at temperature T from the
    teacher's over the places, plus 1 - alpha times the cross entropy with ``labels``.  Places outside the vocabulary (-1) are absent; rows without
    any, and labels outside the vocabulary, contribute nothing.  Gradients go to the logits.  (A program that knows the weight of every row ahead saves
    the second read of the logits with binding.lgn_distill_loss, which forms the gradient with the loss.)"""

    def __init__(self, temperature: float = 1.0, alpha: float = 1.0):
        super().__init__()
        self.temperature, self.alpha = float(temperature), float(alpha)

    def forward(self, logits: torch.Tensor, ids: torch.Tensor, teacher: torch.Tensor, labels: Optional[torch.Tensor] = None) -> torch.Tensor:
        """logits ... x vocab, ids and teacher ... x top, labels ...; the losses have the shape of the rows."""
        shape, top = logits.shape[:-1], ids.shape[-1]
        if ids.shape[:-1] != shape or teacher.shape != ids.shape or (labels is not None and labels.shape != shape):
            raise ValueError("logits, ids, teacher and labels must have the same rows")
        rows = shape.numel()
        flat = None if labels is None else labels.reshape(rows).contiguous()
        loss = _DistillFn.apply(logits.reshape(rows, logits.shape[-1]), _rows(ids.reshape(rows, top)), _rows(teacher.detach().reshape(rows, top)), flat,
                                self.temperature, self.alpha)
        return loss.reshape(shape)


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
