"""The operator-level workflow of Def. 3.1 as a PyTorch autograd function and module.

Forward: the output is exact, the input is compressed and only the compressed form is saved for the
backward pass.  Backward: the input gradient is exact (Thm 3.2.2(a)), the weight gradient is the factored
estimate of Sec. 4, materialised because `weight.grad` is a dense tensor (update strategy (i)), or, with
`factored_grad=True`, left as its two factors for `LowRankAdamW` (update strategy (ii)).

Everything numerical happens in libacc's kernels through `binding`; this file only allocates the output
tensors with torch and keeps the saved factors on the autograd context.  There is no fallback: without the
library, importing `binding` raises.
"""
from __future__ import annotations

import itertools
from typing import Optional

import torch

from . import binding as acc

_CODES = {torch.bfloat16: acc.ACC_BF16, torch.float32: acc.ACC_F32}
_FORMATS = {"e4m3": acc.ACC_ACT8_E4M3, "int8": acc.ACC_ACT8_INT8}   # 8-bit checkpoints


def _workspace(nbytes: int, device):
    return torch.empty(max(int(nbytes), 16), dtype=torch.uint8, device=device)


class CompressedLinearFunction(torch.autograd.Function):
    """y = x @ weight.T (+ bias) with `weight` in torch.nn.Linear's [out_features, in_features] layout.

    compressor "rp": the seeded Gaussian token sketch (unbiased; keeps Xs [in_features, rank] + the seed);
    compressor "rsvd": randomized range finder + projection (keeps U [tokens, rank] and V [in_features, rank]);
    compressor "e4m3" or "int8": an 8-bit checkpoint of the whole input (1 + 1 / 32 bytes per element, `rank` unused), from
    which the weight gradient is formed in full; none is made for a weight that requires no gradient.
    `seed` must differ from call to call for the random projection to be unbiased over a training run.
    Linears that share an input (q/k/v, gate/up; Sec. 5.1) are compressed once by stacking their weights
    into one call.
    """

    @staticmethod
    def forward(ctx, x, weight, bias, rank: int, seed: int, compressor: str = "rp", power_iters: int = 0,
                factor_sink=None):
        if x.dtype not in _CODES or weight.dtype != x.dtype:
            raise TypeError("x and weight must both be bfloat16 or both float32")
        if not x.is_cuda or weight.device != x.device or (bias is not None and bias.device != x.device):
            raise ValueError("x, weight and bias must be on one GPU")
        d_out, d_in = weight.shape
        x2 = x.reshape(-1, d_in)
        if not x2.is_contiguous():
            x2 = x2.contiguous()
        w = weight if weight.is_contiguous() else weight.contiguous()
        n, code, dev = x2.shape[0], _CODES[x.dtype], x.device
        flags = acc.ACC_FLAG_W_OUT_IN
        y = torch.empty(n, d_out, dtype=x.dtype, device=dev)
        if compressor == "rp":
            desc = acc.make_desc(n, d_in, d_out, rank, seed=seed, io_dtype=code, flags=flags)
            xs = torch.empty(d_in, rank, dtype=x.dtype, device=dev)
            acc.acc_linear_fwd(desc, x2, w, y, xs, _workspace(acc.acc_linear_workspace_bytes(desc, False), dev))
            ctx.save_for_backward(w, xs)
        elif compressor == "rsvd":
            desc = acc.make_desc(n, d_in, d_out, rank, seed=seed, io_dtype=code,
                                 flags=flags | (int(power_iters) << acc.ACC_FLAG_RSVD_POWER_SHIFT))
            u = torch.empty(n, rank, dtype=x.dtype, device=dev)
            v = torch.empty(d_in, rank, dtype=x.dtype, device=dev)
            acc.acc_linear_fwd_rsvd(desc, x2, w, y, u, v, _workspace(acc.acc_rsvd_workspace_bytes(desc, False), dev))
            ctx.save_for_backward(w, u, v)
        elif compressor in _FORMATS:
            if factor_sink is not None:
                raise ValueError("an 8-bit checkpoint gives a full weight gradient, not a factored one")
            fmt = _FORMATS[compressor]
            x2, w = _aligned(x2), _aligned(w)
            if ctx.needs_input_grad[1]:
                kept = acc.alloc_act8(acc.make_act8_desc(n, d_in, io_dtype=code, format=fmt), dev)
            else:   # nothing is kept for a weight gradient that nobody forms
                kept, flags = (), flags | acc.ACC_FLAG_SKIP_SKETCH
            if n:
                with torch.cuda.device(dev):
                    acc.acc_linear_fwd_act8(acc.make_desc(n, d_in, d_out, 8, io_dtype=code, flags=flags), fmt, x2, w, y, *(kept or (None, None)))
            ctx.save_for_backward(w, *kept)
        else:
            raise ValueError("compressor must be 'rp', 'rsvd', 'e4m3' or 'int8'")
        if bias is not None:
            y += bias
        ctx.meta = (compressor, n, d_in, d_out, rank, seed, code, bias is not None, x.shape)
        ctx.factor_sink = factor_sink
        return y.reshape(*x.shape[:-1], d_out)

    @staticmethod
    def backward(ctx, dy):
        compressor, n, d_in, d_out, rank, seed, code, has_bias, x_shape = ctx.meta
        dy2 = dy.reshape(n, d_out)
        if not dy2.is_contiguous():
            dy2 = dy2.contiguous()
        dev, dt = dy.device, dy.dtype
        if compressor in _FORMATS:
            return CompressedLinearFunction._backward_act8(ctx, dy2)
        dx = torch.empty(n, d_in, dtype=dt, device=dev)
        gr = torch.empty(d_out, rank, dtype=dt, device=dev)
        sink = ctx.factor_sink
        dw = None if sink is not None else torch.empty(d_out, d_in, dtype=dt, device=dev)
        desc = acc.make_desc(n, d_in, d_out, rank, seed=seed, io_dtype=code, flags=acc.ACC_FLAG_W_OUT_IN)
        if compressor == "rp":
            w, xs = ctx.saved_tensors
            ws = _workspace(acc.acc_linear_workspace_bytes(desc, True), dev)
            acc.acc_linear_bwd(desc, dy2, w, xs, dx, gr, dw, ws)
            left = xs
        else:
            w, u, v = ctx.saved_tensors
            ws = _workspace(max(acc.acc_rsvd_workspace_bytes(desc, True), acc.acc_linear_workspace_bytes(desc, True)), dev)
            acc.acc_linear_bwd_rsvd(desc, dy2, w, u, v, dx, gr, dw, ws)
            left = v
        if sink is not None:   # the weight gradient stays factored: left [d_in, r], gr [d_out, r]
            sink.grad_factors = (left, gr)
        db = None
        if has_bias:
            db = torch.empty(d_out, dtype=dt, device=dev)
            # the backward pass is done with its workspace in stream order, and it is large enough for both
            acc.acc_linear_bias_grad(desc, dy2, db, ws)
        return dx.reshape(x_shape), dw, db, None, None, None, None, None

    @staticmethod
    @torch.autograd.function.once_differentiable
    def _backward_act8(ctx, dy2):
        compressor, n, d_in, d_out, _, _, code, has_bias, x_shape = ctx.meta
        w, *kept = ctx.saved_tensors
        q, e = kept or (None, None)
        dy2 = _aligned(dy2)
        dev, dt = dy2.device, dy2.dtype
        want_dx, want_dw = ctx.needs_input_grad[:2]
        want_db = has_bias and ctx.needs_input_grad[2]
        if n == 0:
            return (dy2.new_empty(x_shape) if want_dx else None, dy2.new_zeros(d_out, d_in) if want_dw else None,
                    dy2.new_zeros(d_out) if want_db else None, None, None, None, None, None)
        desc = acc.make_desc(n, d_in, d_out, 8, io_dtype=code, flags=acc.ACC_FLAG_W_OUT_IN)
        dx = torch.empty(n, d_in, dtype=dt, device=dev) if want_dx else None
        dw = torch.empty(d_out, d_in, dtype=dt, device=dev) if want_dw else None
        db = None
        with torch.cuda.device(dev):
            if want_dx or want_dw:
                ws = _workspace(acc.acc_linear_act8_workspace_bytes(desc), dev) if want_dw else None
                acc.acc_linear_bwd_act8(desc, _FORMATS[compressor], dy2, w, q, e, dx, dw, ws)
            if want_db:
                db = torch.empty(d_out, dtype=dt, device=dev)
                acc.acc_linear_bias_grad(desc, dy2, db, _workspace(acc.acc_linear_workspace_bytes(desc, True), dev))
        return None if dx is None else dx.reshape(x_shape), dw, db, None, None, None, None, None


class CompressedLinear(torch.nn.Module):
    """Drop-in for torch.nn.Linear (same parameter names and layout) that keeps only the compressed input
    for the backward pass.  Each forward call draws a fresh sketch seed from a per-module counter.  `rank` is that of the
    "rp" and "rsvd" compressors, which need one; "e4m3" and "int8" have none."""

    def __init__(self, in_features: int, out_features: int, rank: Optional[int] = None, bias: bool = True, compressor: str = "rp",
                 seed: int = 0, power_iters: int = 0, device=None, dtype=torch.bfloat16, factored_grad: bool = False):
        super().__init__()
        if compressor not in _FORMATS:
            if rank is None:
                raise TypeError(f"compressor '{compressor}' needs a rank")
            if rank <= 0:
                raise ValueError("rank must be positive")
        self.factored_grad = factored_grad
        self.grad_factors = None   # (left [in, rank], gr [out, rank]) of the last backward pass when factored_grad
        self.in_features, self.out_features, self.rank = in_features, out_features, rank or 0
        self.compressor, self.power_iters = compressor, power_iters
        self.weight = torch.nn.Parameter(torch.empty(out_features, in_features, device=device, dtype=dtype))
        if bias:
            self.bias = torch.nn.Parameter(torch.zeros(out_features, device=device, dtype=dtype))
        else:
            self.register_parameter("bias", None)
        torch.nn.init.normal_(self.weight, std=0.02)
        self._seeds = itertools.count(int(seed) << 20)

    def forward(self, x):
        # (the function sees its weight's requires_grad, not whether gradients are recorded at all)
        weight = self.weight if torch.is_grad_enabled() else self.weight.detach()
        return CompressedLinearFunction.apply(x, weight, self.bias, self.rank, next(self._seeds),
                                              self.compressor, self.power_iters,
                                              self if self.factored_grad else None)

    def extra_repr(self):
        return (f"in_features={self.in_features}, out_features={self.out_features}, rank={self.rank}, "
                f"compressor={self.compressor}, bias={self.bias is not None}")


def _aligned(t):
    """t, contiguous and 16-byte aligned: a slice of a vector (labels[1:]) is the one and not the other."""
    t = t.contiguous()
    return t.clone() if t.data_ptr() % 16 else t


def _rows(t, width):
    """t as rows of `width` elements the library can take as they lie (16-byte aligned, any stride), else a copy."""
    t2 = t.reshape(-1, width)
    if t2.stride(1) != 1 or (t2.shape[0] > 1 and (t2.stride(0) % 8 or not width <= t2.stride(0) <= 1 << 18)) or t2.data_ptr() % 16:
        t2 = _aligned(t2)
    return t2


def _ld(t2):
    return t2.stride(0) if t2.shape[0] > 1 else 0


class CompressedSwiGLUFunction(torch.autograd.Function):
    """silu(gate) * up of the two halves of x [..., 2 f] (gate first); gate and up are kept as 8-bit checkpoints, half of
    x's bytes in bfloat16, and the gradients are formed from those (acc_gated_fwd_act8 / acc_gated_bwd_act8)."""

    @staticmethod
    def forward(ctx, x, fmt: str = "int8"):
        if x.dtype not in _CODES:
            raise TypeError("x must be bfloat16 or float32")
        if fmt not in _FORMATS:
            raise ValueError("format must be 'e4m3' or 'int8'")
        f = x.shape[-1] // 2
        if x.shape[-1] != 2 * f:
            raise ValueError("the last dimension holds gate and up: it must be even")
        x2 = _rows(x, 2 * f)
        n, dev = x2.shape[0], x.device
        h = torch.empty(n, f, dtype=x.dtype, device=dev)
        ctx.meta = (n, f, fmt, x.shape)
        if n == 0:
            return h.reshape(*x.shape[:-1], f)
        desc = acc.make_gated_desc(n, f, ldg=x2.stride(0) if n > 1 else 2 * f, io_dtype=_CODES[x.dtype], format=_FORMATS[fmt])
        kept = acc.alloc_gated_act8(desc, dev)
        with torch.cuda.device(dev):
            acc.acc_gated_fwd_act8(desc, x2[:, :f], x2[:, f:], h, *kept)
        ctx.save_for_backward(*kept)
        return h.reshape(*x.shape[:-1], f)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dh):
        n, f, fmt, shape = ctx.meta
        dx = torch.empty(n, 2 * f, dtype=dh.dtype, device=dh.device)
        if n:
            dh2 = _rows(dh, f)
            desc = acc.make_gated_desc(n, f, ldg=2 * f, ldh=_ld(dh2), io_dtype=_CODES[dh.dtype], format=_FORMATS[fmt])
            with torch.cuda.device(dh.device):
                acc.acc_gated_bwd_act8(desc, dh2, *ctx.saved_tensors, dx[:, :f], dx[:, f:])
        return dx.reshape(shape), None


class CompressedSwiGLU(torch.nn.Module):
    """The gated activation of an MLP whose gate and up projections are one linear: [..., 2 f] -> [..., f]."""

    def __init__(self, format: str = "int8"):
        super().__init__()
        if format not in _FORMATS:
            raise ValueError("format must be 'e4m3' or 'int8'")
        self.format = format

    def forward(self, x):
        return CompressedSwiGLUFunction.apply(x, self.format)

    def extra_repr(self):
        return f"format={self.format}"


class LinearCrossEntropyFunction(torch.autograd.Function):
    """Per-token softmax cross entropy (float32) of x @ weight.T against `target`, weight [vocabulary, features], without the
    logits (acc_linear_ce_fwd / acc_linear_ce_bwd).  Kept for the backward pass: x, weight, target and two floats a token.
    Negative targets have no loss and no gradient, those beyond the vocabulary a loss of NaN and no gradient.  With bfloat16
    tensors the logits' gradient is rounded to bfloat16 before its products with weight and x; logits, losses and all sums are
    float32."""

    @staticmethod
    def forward(ctx, x, weight, target):
        if x.dtype not in _CODES or weight.dtype != x.dtype:
            raise TypeError("x and weight must both be bfloat16 or both float32")
        if target.dtype != torch.int64 or target.shape != x.shape[:-1]:
            raise TypeError("target must be int64, one per token")
        if not (x.device == weight.device == target.device):
            raise ValueError("x, weight and target must be on one device")
        v, d = weight.shape
        if x.shape[-1] != d:
            raise ValueError(f"x has {x.shape[-1]} features, weight {d}")
        x2, w, t = _rows(x, d), _rows(weight, d), _aligned(target.reshape(-1))
        n, dev = x2.shape[0], x.device
        loss = torch.empty(n, dtype=torch.float32, device=dev)
        ctx.meta = (n, d, v, x.shape)
        if n == 0:
            ctx.save_for_backward(w)
            return loss.reshape(target.shape)
        stats = torch.empty(2, n, dtype=torch.float32, device=dev)
        desc = LinearCrossEntropyFunction._desc(ctx, x2, w)
        with torch.cuda.device(dev):
            acc.acc_linear_ce_fwd(desc, x2, w, t, loss, stats, _workspace(acc.acc_linear_ce_workspace_bytes(desc, False), dev))
        ctx.save_for_backward(w, x2, t, stats)
        return loss.reshape(target.shape)

    @staticmethod
    def _desc(ctx, x2, w):
        n, d, v, _ = ctx.meta
        return acc.make_ce_desc(n, d, v, ldx=_ld(x2), ldw=_ld(w), io_dtype=_CODES[w.dtype])

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss):
        n, d, v, shape = ctx.meta
        want_dx, want_dw = ctx.needs_input_grad[:2]
        w, dev = ctx.saved_tensors[0], dloss.device
        if n == 0 or not (want_dx or want_dw):
            return (torch.empty(shape, dtype=w.dtype, device=dev) if want_dx else None,
                    torch.zeros(v, d, dtype=w.dtype, device=dev) if want_dw else None, None)
        _, x2, t, stats = ctx.saved_tensors
        if want_dx:   # the call has one row stride for x and dx: dense rows of both, or the gradient would hold the gaps too
            x2 = x2.contiguous()
        desc = LinearCrossEntropyFunction._desc(ctx, x2, w)
        g = _aligned(dloss.reshape(-1).to(torch.float32))
        dx = torch.empty(n, d, dtype=w.dtype, device=dev) if want_dx else None
        dw = torch.empty(v, d, dtype=w.dtype, device=dev) if want_dw else None
        with torch.cuda.device(dev):
            acc.acc_linear_ce_bwd(desc, x2, w, t, stats, g, dx, dw, _workspace(acc.acc_linear_ce_workspace_bytes(desc, True), dev))
        return None if dx is None else dx.reshape(shape), dw, None


class LinearCrossEntropy(torch.nn.Module):
    """The last product of a language model with its loss: torch.nn.Linear(features, vocabulary, bias=False) followed by
    torch.nn.functional.cross_entropy, without the logits.  `weight` may be tied to an embedding table's.

    reduction "mean" (over the tokens whose target is not ignore_index), "sum" or "none"."""

    def __init__(self, in_features: int, vocabulary: int, ignore_index: int = -100, reduction: str = "mean", device=None,
                 dtype=torch.bfloat16):
        super().__init__()
        if reduction not in ("mean", "sum", "none"):
            raise ValueError("reduction must be 'mean', 'sum' or 'none'")
        self.ignore_index, self.reduction = ignore_index, reduction
        self.weight = torch.nn.Parameter(torch.empty(vocabulary, in_features, device=device, dtype=dtype))
        torch.nn.init.normal_(self.weight, std=0.02)

    def forward(self, x, target):
        if self.ignore_index >= 0:
            target = torch.where(target == self.ignore_index, -1, target)
        loss = LinearCrossEntropyFunction.apply(x, self.weight, target)
        if self.reduction == "none":
            return loss
        total = loss.sum()
        return total if self.reduction == "sum" else total / (target >= 0).sum()

    def extra_repr(self):
        return f"in_features={self.weight.shape[1]}, vocabulary={self.weight.shape[0]}, reduction={self.reduction}"


class LowRankAdamW:
    """Update strategy (ii) of Sec. 4 for `CompressedLinear(..., factored_grad=True)` modules: AdamW whose moments
    have the shape [out_features, proj_rank]; the weights are updated in place by acc_lowrank_adamw_step, and no
    dense gradient or dense optimizer state is ever allocated.

    proj_rank > 0: moments live in the range of a projector [in_features, proj_rank] computed from the factored
    gradient by acc_lowrank_projector and refreshed every `proj_gap` steps (the moments are kept across a
    refresh).  proj_rank = 0: the left factor of each step is its own projector.  One backward pass per step
    (factors of several micro-batches cannot be summed).  Biases are left to an ordinary optimizer.
    """

    def __init__(self, modules, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.0,
                 scale: float = 1.0, proj_rank: int = 0, proj_gap: int = 200, seed: int = 0):
        self.modules = [m for m in modules if isinstance(m, CompressedLinear) and m.factored_grad]
        if not self.modules:
            raise ValueError("no CompressedLinear module with factored_grad=True")
        self.lr, self.betas, self.eps, self.weight_decay, self.scale = lr, betas, eps, weight_decay, scale
        self.proj_rank, self.proj_gap, self.seed = int(proj_rank), int(proj_gap), int(seed)
        self.state = {}

    @torch.no_grad()
    def step(self):
        k = self.proj_rank
        for idx, m in enumerate(self.modules):
            if m.grad_factors is None:
                continue
            left, gr = m.grad_factors
            w = m.weight.data
            if not w.is_contiguous():
                raise ValueError("weight must be contiguous to be updated in place")
            st = self.state.get(m)
            if st is None:
                rows = k if k else m.rank
                st = self.state[m] = {
                    "step": 0,
                    "exp_avg": torch.zeros(m.out_features, rows, dtype=torch.float32, device=gr.device),
                    "exp_avg_sq": torch.zeros(m.out_features, rows, dtype=torch.float32, device=gr.device),
                    "projector": torch.empty(m.in_features, k, dtype=gr.dtype, device=gr.device) if k else None}
            refresh = k and st["step"] % self.proj_gap == 0
            st["step"] += 1
            # a fresh range-finder seed per module and refresh
            desc = acc.make_desc(1, m.in_features, m.out_features, m.rank, io_dtype=_CODES[w.dtype],
                                 factor_dtype=_CODES[gr.dtype], flags=acc.ACC_FLAG_W_OUT_IN,
                                 seed=(self.seed << 40) + (idx << 24) + st["step"] // max(self.proj_gap, 1))
            ws = _workspace(acc.acc_lowrank_workspace_bytes(desc, k), gr.device)
            if refresh:
                acc.acc_lowrank_projector(desc, k, left, gr, st["projector"], ws)
            hyper = acc.make_hyper(st["step"], self.lr, self.betas[0], self.betas[1], self.eps, self.weight_decay,
                                   self.scale)
            acc.acc_lowrank_adamw_step(desc, hyper, st["projector"], k, left, gr, st["exp_avg"], st["exp_avg_sq"],
                                       w, ws)
            m.grad_factors = None

    def zero_grad(self):
        for m in self.modules:
            m.grad_factors = None
