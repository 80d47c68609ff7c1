"""Drop-in PyTorch layers over the C ABI (the way the paper ships its kernels: App. F).

Only what is stashed for backward differs from the stock layers:
  InplaceGELU        keeps the output (which the next Linear keeps anyway) and a 1-bit mask
  InplaceSiLU        the same for SiLU (Sec. 5.1)
  InplaceLayerNorm   keeps the output and one float per row
  TempoAttentionCore softmax -> dropout -> (. @ V) keeping the softmax output P and a 1-bit
                     mask; the dropout output is a transient in forward and is recomputed by
                     the backward kernel for the gradient of V (Sec. 3.3).
  RotaryPositions    turns the heads of q and k by their positions, on one axis or several; keeps nothing but those
  TempoWindowAttention  attention with a sliding window and first tokens that stay visible, over no matrix of scores: keeps q, k, v,
                     its output and one float per row
  TempoResidualNorm  the place between two blocks: a norm of the block's output, its gate, the residual and the next block's norm, from
                     the block's output, the residual and two floats per norm and row
  TempoGatedFFN      a gated feed-forward block keeping its input and the two projections; their
                     activated product, which the second Linear would keep, is made once more by
                     the backward kernel
  TempoEncoderLayer  an encoder layer of the first three: in float32 one native call each way on HIP
                     kernels alone where nothing else can see its parts, else those parts; with
                     rotary positions or a gated feed-forward block in it on request
Every arithmetic step of these layers runs in the HIP kernels; the matrix products around
them, where the layer is made of its parts, are ordinary library GEMMs (torch.matmul, nn.Linear).
"""
from __future__ import annotations

import math
from typing import Optional, Tuple

import torch
import torch.nn.functional as F
from torch import nn
from torch.autograd import forward_ad
from torch.nn.modules import linear, module

from . import binding as B


def _words(n: int, device) -> torch.Tensor:
    return torch.empty(B.mask_words(n), dtype=torch.int32, device=device)


# `made`, in the three functions below: what the forward has already made, which is then not run (x and scores give only their
# place in the graph).

class _InplaceGELUFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, kind, made):
        if made is None:
            x = x.contiguous()
            y = torch.empty_like(x)
            mask = _words(x.numel(), x.device)
            if kind == "silu":
                B.tempo_silu_fwd(x, y, mask)
            else:
                B.tempo_gelu_fwd(x, y, mask, kind)
        else:
            y, mask = made[0].detach(), made[1]
        ctx.kind = kind
        ctx.save_for_backward(y, mask)
        return y

    @staticmethod
    def backward(ctx, dy):
        y, mask = ctx.saved_tensors
        dy = dy.contiguous()
        dx = torch.empty_like(dy)
        if ctx.kind == "silu":
            B.tempo_silu_bwd(dy, y, mask, dx)
        else:
            B.tempo_gelu_bwd(dy, y, mask, dx, ctx.kind)
        return dx, None, None


class InplaceGELU(nn.Module):
    """GELU whose backward needs the output and one bit per element (Sec. 3.1)."""

    def __init__(self, approximate: str = "none"):
        super().__init__()
        self.kind = {"none": "erf", "tanh": "tanh"}[approximate]

    def forward(self, x):
        return _InplaceGELUFn.apply(x, self.kind, None)


class InplaceSiLU(nn.Module):
    """SiLU with the same stash as InplaceGELU: the in-place recipe for elementwise layers
    (Sec. 5.1) on another activation with a single minimum."""

    def forward(self, x):
        return _InplaceGELUFn.apply(x, "silu", None)


class _InplaceLayerNormFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gamma, beta, eps, made):
        if made is None:
            x = x.contiguous()
            M = x.shape[-1]
            N = x.numel() // M
            y = torch.empty_like(x)
            rstd = torch.empty(N, dtype=torch.float32, device=x.device)
            B.tempo_layernorm_fwd(x, gamma, beta, y, rstd, None, eps)
        else:
            y, rstd = made[0].detach(), made[1]
        ctx.save_for_backward(y, gamma, beta, rstd)
        return y

    @staticmethod
    def backward(ctx, dy):
        y, gamma, beta, rstd = ctx.saved_tensors
        dy = dy.contiguous()
        M = y.shape[-1]
        N = y.numel() // M
        dx = torch.empty_like(dy)
        dgamma = torch.empty_like(gamma)
        dbeta = torch.empty_like(beta)
        ws = torch.empty(B.tempo_layernorm_bwd_workspace_bytes(N, M), dtype=torch.uint8,
                         device=y.device)
        B.tempo_layernorm_bwd(dy, y, gamma, beta, rstd, dx, dgamma, dbeta, ws)
        return dx, dgamma, dbeta, None, None


class _Float32Parameters(nn.Module):
    def _apply(self, fn, recurse=True):
        # .bfloat16() / .half() / .to(dtype) on a model must not narrow gamma and beta: the
        # kernels read them as float32.  Follow the device of the cast, keep the values.
        def keep_float32(t):
            out = fn(t)
            if t.dtype == torch.float32 and out.dtype != torch.float32:
                out = t.to(device=out.device)
            return out
        return super()._apply(keep_float32, recurse)


class InplaceLayerNorm(_Float32Parameters):
    """LayerNorm over the last dimension whose backward needs the output and rstd (Sec. 3.2).
    Parameters are float32 whatever the activation dtype; gamma must stay non-zero."""

    def __init__(self, hidden: int, eps: float = 1e-5):
        super().__init__()
        self.weight = nn.Parameter(torch.ones(hidden, dtype=torch.float32))
        self.bias = nn.Parameter(torch.zeros(hidden, dtype=torch.float32))
        self.eps = eps

    def forward(self, x):
        w, b = self.weight, self.bias
        if w.dtype != torch.float32 or b.dtype != torch.float32:   # parameters replaced by hand
            w, b = w.float(), b.float()
        return _InplaceLayerNormFn.apply(x, w, b, self.eps, None)


class _AttentionCoreFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, scores, v, key_len, causal, p, seed, offset, store_mask, made):
        if made is None:
            scores = scores.contiguous()
            probs = torch.empty_like(scores)
            out = torch.empty_like(scores)      # transient: freed when forward returns
            keep = _words(scores.numel(), scores.device)
            B.tempo_attn_softmax_dropout_fwd(scores, key_len, causal, probs, out, keep, p, seed, offset)
        else:
            probs, keep = made[:2]
        ctx.rng = (p, seed, offset)
        ctx.store_mask = store_mask
        if store_mask:
            ctx.save_for_backward(probs, v, keep)
        else:                                   # the mask is a transient too: drawn again later
            ctx.save_for_backward(probs, v)
        return torch.matmul(out, v) if made is None else made[2].detach()

    @staticmethod
    def backward(ctx, dctx):
        probs, v = ctx.saved_tensors[:2]
        dout = torch.matmul(dctx, v.transpose(-1, -2)).contiguous()
        out_re = torch.empty_like(probs)
        dscores = torch.empty_like(probs)
        p, seed, offset = ctx.rng
        if ctx.store_mask:
            B.tempo_attn_softmax_dropout_bwd(dout, probs, ctx.saved_tensors[2], dscores, out_re, p)
        else:
            B.tempo_attn_softmax_dropout_bwd_regen(dout, probs, dscores, out_re, p, seed, offset)
        dv = torch.matmul(out_re.transpose(-1, -2), dctx)
        return (dscores, dv) + (None,) * 7


class TempoAttentionCore(nn.Module):
    """context = dropout(softmax(mask(scores))) @ V for scores [B, A, Sq, Sk] already scaled by
    1/sqrt(d).  Each forward in training mode draws a fresh mask: the counter offset advances.
    store_mask=False keeps no mask for backward, which then draws the same bits again."""

    def __init__(self, p: float = 0.1, seed: int = 0x5EED, store_mask: bool = True):
        super().__init__()
        self.p, self.seed, self.offset, self.store_mask = p, seed, 0, store_mask

    def forward(self, scores, v, key_len=None, causal=False):
        p = self.p if self.training else 0.0
        self.offset += 1
        return _AttentionCoreFn.apply(scores, v, key_len, causal, p, self.seed, self.offset,
                                      self.store_mask, None)


def rotary_frequencies(dim: int, base: float = 10000.0, scaling: Optional[str] = None, factor: float = 1.0,
                       trained: int = 0, turns: Tuple[float, float] = (1.0, 32.0)):
    """The dim / 2 frequencies base^(-2 i / dim) of rotary positions in float64, radians per position, and what q and k are
    scaled by.  scaling, for contexts `factor` times as long as the trained one:
      "linear"  positions are factor times closer;
      "base"    the base grows by factor^(dim / (dim - 2)): the slowest frequency is divided by factor, the fastest left;
      "parts"   frequencies that make fewer than turns[0] turns in the `trained` positions are divided by factor, those that
                make more than turns[1] are left, with a linear ramp between; q and k are scaled by 0.1 ln(factor) + 1."""
    if dim < 2 or dim % 2:
        raise ValueError(f"dim must be even and positive, got {dim}")
    if not (base > 0 and factor >= 1.0):
        raise ValueError(f"base must be positive and factor at least 1, got {base} and {factor}")
    if scaling == "base":
        if dim == 2:
            raise ValueError("scaling the base needs more than one frequency")
        base *= factor ** (dim / (dim - 2))
    f = base ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)
    if scaling in (None, "base"):
        return f, 1.0
    if scaling == "linear":
        return f / factor, 1.0
    if scaling != "parts":
        raise ValueError(f'scaling must be None, "linear", "base" or "parts", got {scaling!r}')
    if trained < 1 or not turns[0] < turns[1]:
        raise ValueError(f"trained must be positive and turns ascending, got {trained} and {turns}")
    left = ((trained * f / (2 * math.pi) - turns[0]) / (turns[1] - turns[0])).clamp(0.0, 1.0)
    return f * (left + (1.0 - left) / factor), 0.1 * math.log(factor) + 1.0


class _RotaryFn(torch.autograd.Function):
    """q and k [B, S, heads, D], either of which may be None, to tensors that lie by head.  Linear: the gradient is the turn the
    other way, which is differentiable in turn."""

    @staticmethod
    def forward(ctx, q, k, freqs, positions, start, layout, scale, back, axes=None):
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(freqs, positions, axes)
        ctx.setting = start, layout, scale, back
        sides = [None if t is None else t if t.stride(-1) == 1 else t.contiguous() for t in (q, k)]
        out = [None if t is None else t.new_empty(t.shape[0], t.shape[2], t.shape[1], t.shape[3]).transpose(1, 2) for t in sides]
        first, second = (0, 1) if q is not None else (1, 0)
        if axes is None:
            call, where = B.tempo_rotary_bwd if back else B.tempo_rotary_fwd, (positions,)
        else:
            call, where = B.tempo_rotary_axes_bwd if back else B.tempo_rotary_axes_fwd, (axes, positions)
        call(sides[first], sides[second], freqs, *where, out[first], out[second], layout, scale, start)
        return tuple(out)

    @staticmethod
    def backward(ctx, dq, dk):
        start, layout, scale, back = ctx.setting
        freqs, positions, axes = ctx.saved_tensors
        dq, dk = (g if n else None for g, n in zip((dq, dk), ctx.needs_input_grad))
        if dq is not None or dk is not None:
            dq, dk = _RotaryFn.apply(dq, dk, freqs, positions, start, layout, scale, not back, axes)
        return dq, dk, None, None, None, None, None, None, None


def rotary_axes(sections: Tuple[int, ...], order: str = "blocks") -> torch.Tensor:
    """Which axis each pair turns by (uint8), sections[a] of them by axis a: "blocks" of pairs, or "cyclic", dealt out in turn to the axes
    that have not got theirs."""
    if not 1 <= len(sections) <= 4 or min(sections) < 0 or sum(sections) < 1:
        raise ValueError(f"sections are of 1 to 4 axes and not all empty, got {sections}")
    if order == "blocks":
        of_pairs = [a for a, n in enumerate(sections) for _ in range(n)]
    elif order == "cyclic":
        of_pairs = [a for turn in range(max(sections)) for a, n in enumerate(sections) if turn < n]
    else:
        raise ValueError(f'order must be "blocks" or "cyclic", got {order!r}')
    return torch.tensor(of_pairs, dtype=torch.uint8)


class RotaryPositions(nn.Module):
    """Rotary positions of q and k [B, heads, S, D], of any strides, whose numbers of heads may differ; k may be None.  positions:
    [S] or [B, S], int32 or int64 (0, 1, ... if None); start is added to them.  Turns the first `dim` elements of a head; layout:
    "half" pairs element i with i + dim / 2, "interleaved" 2 i with 2 i + 1.  sections, order: rotary_axes()'s, for several axes (time,
    height and width); positions are [axes, S] or [axes, B, S] then.  own: each axis has all frequencies of its own pairs' number, not its
    part of one row of them.  The other arguments are rotary_frequencies()'s."""

    def __init__(self, dim: int, base: float = 10000.0, layout: str = "half", scaling: Optional[str] = None, factor: float = 1.0,
                 trained: int = 0, turns: Tuple[float, float] = (1.0, 32.0), sections: Optional[Tuple[int, ...]] = None,
                 order: str = "blocks", own: bool = False):
        super().__init__()
        if layout not in ("half", "interleaved"):
            raise ValueError(f'layout must be "half" or "interleaved", got {layout!r}')
        freqs, self.scale = rotary_frequencies(dim, base, scaling, factor, trained, turns)
        self.layout, axes = layout, None
        self.n_axes = 0 if sections is None else len(sections)
        if sections is not None:
            axes = rotary_axes(sections, order)
            if axes.numel() != dim // 2:
                raise ValueError(f"sections must make {dim // 2} pairs, got {sections}")
            if own:
                for a, n in enumerate(sections):
                    if n > 0:
                        freqs[axes == a] = rotary_frequencies(2 * n, base, scaling, factor, trained, turns)[0]
        elif own:
            raise ValueError("own frequencies are those of sections' axes")
        self.register_buffer("freqs", freqs, persistent=False)
        self.register_buffer("axes", axes, persistent=False)

    def _apply(self, fn, recurse=True):
        # a cast of the model follows the device and leaves the frequencies in float64
        freqs, axes = self.freqs, self.axes
        super()._apply(fn, recurse)
        if self.freqs.dtype != torch.float64:
            self.freqs = freqs.to(device=self.freqs.device)
        if axes is not None and self.axes.dtype != torch.uint8:
            self.axes = axes.to(device=self.axes.device)
        return self

    def forward(self, q, k=None, positions=None, start: int = 0):
        if self.axes is not None and (positions is None or positions.dim() < 2 or positions.shape[0] != self.n_axes):
            raise ValueError(f"{self.n_axes} axes have positions, [{self.n_axes}, S] or [{self.n_axes}, B, S], got "
                             f"{None if positions is None else tuple(positions.shape)}")
        k_in = None if k is None else k.transpose(1, 2)
        q, k = _RotaryFn.apply(q.transpose(1, 2), k_in, self.freqs, positions, start, self.layout, self.scale, False, self.axes)
        return q.transpose(1, 2), None if k is None else k.transpose(1, 2)


class _WindowAttentionFn(torch.autograd.Function):
    """q [B, Sq, heads, D], k and v [B, Sk, kv_heads, D] to an output that lies by token."""

    @staticmethod
    def forward(ctx, q, k, v, window, sinks, scale, key_len, query_start, keep):
        q, k, v = (t if t.stride(-1) == 1 else t.contiguous() for t in (q, k, v))
        out = q.new_empty(q.shape)
        lse = q.new_empty(q.shape[0], q.shape[2], q.shape[1], dtype=torch.float32) if keep else None
        B.tempo_window_attn_fwd(q, k, v, out, lse, window, sinks, scale, key_len, query_start)
        ctx.setting = window, sinks, scale
        if keep:
            ctx.save_for_backward(q, k, v, out, lse, key_len, query_start)
        return out

    @staticmethod
    def backward(ctx, dout):
        if torch.is_grad_enabled():      # the kernels' gradients would be constants to a second derivative
            raise RuntimeError("TempoWindowAttention has no second derivative: its gradients cannot be taken with create_graph=True")
        q, k, v, out, lse, key_len, query_start = ctx.saved_tensors
        dout = dout if dout.stride(-1) == 1 else dout.contiguous()
        dq, dk, dv = (t.new_empty(t.shape) for t in (q, k, v))
        B.tempo_window_attn_bwd(dout, q, k, v, out, lse, dq, dk, dv, *ctx.setting[:2], ctx.setting[2], key_len, query_start)
        return tuple(g if n else None for g, n in zip((dq, dk, dv), ctx.needs_input_grad)) + (None,) * 6


class TempoWindowAttention(nn.Module):
    """Attention of q [B, heads, Sq, D] over k and v [B, kv_heads, Sk, D], of any strides: a query at position P sees the keys up to P that
    are among the last `window` or the first `sinks`.  Heads of q share those of k and v where there are more of them.  key_len [B]
    int32: keys from there on do not exist; query_start [B] int32: positions of the first queries (Sk - Sq if None), as for new tokens
    of sequences in a cache.  scale: D^-0.5 if None.  No dropout, no second derivative."""

    def __init__(self, window: int, sinks: int = 0, scale: Optional[float] = None):
        super().__init__()
        if window < 1 or sinks < 0:
            raise ValueError(f"window must be at least 1 and sinks at least 0, got {window} and {sinks}")
        if scale is not None and not 0.0 < scale < math.inf:
            raise ValueError(f"scale must be positive and finite, got {scale}")
        self.window, self.sinks, self.scale = window, sinks, scale

    def forward(self, q, k, v, key_len=None, query_start=None):
        if torch.is_autocast_enabled("cuda"):    # as a product would take them
            q, k, v = (t.to(torch.get_autocast_dtype("cuda")) for t in (q, k, v))
        keep = torch.is_grad_enabled() and any(t.requires_grad for t in (q, k, v))
        q, k, v = (t.transpose(1, 2) for t in (q, k, v))
        return _WindowAttentionFn.apply(q, k, v, self.window, self.sinks, self.scale, key_len, query_start, keep).transpose(1, 2)


class _ResidualNormFn(torch.autograd.Function):
    """y = alpha x + beta gate post(f) and h = pre(y), or y alone."""

    @staticmethod
    def forward(ctx, x, f, gate, pw, pb, qw, qb, post, pre, alpha, beta, eps):
        x, f = _aligned(x), _aligned(f)
        M = x.shape[-1]
        rows = x.numel() // M if M else 0
        y, h = torch.empty_like(x), torch.empty_like(x) if pre else None
        stats = [x.new_empty(rows, 2, dtype=torch.float32) if kind else None for kind in (post, pre)]
        B.tempo_residual_norm_fwd(x, f, gate, y, h, post, pw, pb, stats[0], pre, qw, qb, stats[1], alpha, beta, eps, eps)
        ctx.setting = post, pre, alpha, beta
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(f, y if pre else None, gate, pw, pb, qw, *stats)
        return (y, h) if pre else y

    @staticmethod
    def backward(ctx, dy, dh=None):
        if torch.is_grad_enabled():      # the kernels' gradients would be constants to a second derivative
            raise RuntimeError("TempoResidualNorm has no second derivative: its gradients cannot be taken with create_graph=True")
        post, pre, alpha, beta = ctx.setting
        f, y, gate, pw, pb, qw, post_stats, pre_stats = ctx.saved_tensors
        if dy is None and dh is None:
            return (None,) * 12
        if pre and dh is None:
            dh = torch.zeros_like(f)
        dx, df = torch.empty_like(f), torch.empty_like(f)
        need = ctx.needs_input_grad
        like = [torch.empty_like(t) if n else None for t, n in zip((gate, pw, pb, qw), need[2:6])]
        dqb = f.new_empty(f.shape[-1], dtype=torch.float32) if need[6] else None
        B.tempo_residual_norm_bwd(_aligned(dy), _aligned(dh), f, y, gate, dx, df, like[0], post, pw, pb, post_stats, like[1], like[2], pre, qw,
                                  pre_stats, like[3], dqb, alpha, beta)
        return (dx if need[0] else None, df if need[1] else None, *like, dqb) + (None,) * 5


class TempoResidualNorm(_Float32Parameters):
    """The place between two blocks of a pre-norm model, for the residual x and a block's output f: y = alpha x + beta gate post(f), the next
    residual, and h = pre(y), the next block's input (None without a pre).  post, pre: "rms", "layer" or None.  gate: a learned one of
    `hidden` elements that begins at that value; or None, and forward takes one, [hidden] or one for each of equally many rows
    (as [B, hidden] or [B, 1, hidden] beside [B, S, hidden]), or none.  affine: the norms have weights, and with "layer" biases.  Parameters and gates
    are float32 whatever the activation dtype.  No second derivative."""

    def __init__(self, hidden: int, post: Optional[str] = None, pre: Optional[str] = "rms", gate: Optional[float] = None, alpha: float = 1.0,
                 beta: float = 1.0, eps: float = 1e-5, affine: bool = True):
        super().__init__()
        for name, kind in (("post", post), ("pre", pre)):
            if kind not in (None, "rms", "layer"):
                raise ValueError(f'{name} must be "rms", "layer" or None, got {kind!r}')
            weight = nn.Parameter(torch.ones(hidden)) if kind and affine else None
            self.register_parameter(name + "_weight", weight)
            self.register_parameter(name + "_bias", nn.Parameter(torch.zeros(hidden)) if kind == "layer" and affine else None)
        self.register_parameter("gate", None if gate is None else nn.Parameter(torch.full((hidden,), float(gate))))
        self.hidden, self.post, self.pre, self.alpha, self.beta, self.eps = hidden, post, pre, alpha, beta, eps

    def _gate_of_groups(self, gate, x):
        """[hidden] or [groups, hidden], the groups being of x's first dimensions; with as many dimensions as x it has x's sizes first, then
        ones."""
        if gate.dim() == x.dim() > 2:
            first = 0
            while first < x.dim() - 1 and gate.shape[first] == x.shape[first]:
                first += 1
            if all(n == 1 for n in gate.shape[first:-1]):
                return gate.reshape(-1, gate.shape[-1])
        elif gate.dim() == 1 or (gate.dim() == 2 and (x.dim() == 2 or gate.shape[0] in [x.shape[:n].numel() for n in range(x.dim())])):
            return gate
        raise ValueError(f"gate must be [{self.hidden}], [groups, {self.hidden}] for groups of x's first dimensions or like x with ones behind them, "
                         f"got {tuple(gate.shape)} beside {tuple(x.shape)}")

    def forward(self, x, f, gate=None):
        if torch.is_autocast_enabled("cuda"):
            f = f.to(x.dtype)       # a block's output beside a residual in float32
        if x.shape[-1:] != (self.hidden,) or f.shape != x.shape:
            raise ValueError(f"x and f must be [..., {self.hidden}], got {tuple(x.shape)} and {tuple(f.shape)}")
        if gate is not None and self.gate is not None:
            raise ValueError("this place has a gate of its own")
        gate = self.gate if gate is None else gate
        if gate is not None:
            gate = self._gate_of_groups(gate, x).float().contiguous()
        params = [None if p is None else p.float() for p in (self.post_weight, self.post_bias, self.pre_weight, self.pre_bias)]
        out = _ResidualNormFn.apply(x, f, gate, *params, self.post, self.pre, self.alpha, self.beta, self.eps)
        return out if self.pre else (out, None)


def _aligned(t):
    """t as the kernels take it: contiguous, from a multiple of 16 bytes on."""
    if t is None:
        return None
    t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


class _GatedFFNFn(torch.autograd.Function):
    """y = (act(g) u) wd^T + bd, [g | u] = x w^T + b: keeps x and [g | u]."""

    @staticmethod
    def forward(ctx, x, w, b, wd, bd, kind, keep):
        x, w, b = _aligned(x), _aligned(w), _aligned(b)
        ffn = w.shape[0] // 2
        h = x.new_empty(*x.shape[:-1], ffn)      # transient: made once more by the backward
        gu = x.new_empty(*x.shape[:-1], 2 * ffn) if keep else None
        B.tempo_glu_fwd(x, w, b, gu, h, kind)
        ctx.kind = kind
        if keep:
            ctx.save_for_backward(x, w, wd, gu)
        return F.linear(h, wd, bd)

    @staticmethod
    def backward(ctx, dy):
        if torch.is_grad_enabled():      # the kernels' gradients would be constants to a second derivative
            raise RuntimeError("TempoGatedFFN has no second derivative: its gradients cannot be taken with create_graph=True")
        x, w, wd, gu = ctx.saved_tensors
        need = ctx.needs_input_grad
        rows = dy.reshape(-1, dy.shape[-1])
        inner = need[0] or need[1] or need[2]
        h = gu.new_empty(rows.shape[0], wd.shape[1]) if need[3] else None
        dx = torch.empty_like(x) if need[0] else None
        dw = torch.empty_like(w) if need[1] else None
        db = w.new_empty(w.shape[0]) if need[2] else None
        if inner or need[3]:
            dh = torch.matmul(rows, wd) if inner else gu.new_zeros(rows.shape[0], wd.shape[1])
            B.tempo_glu_bwd(_aligned(dh), gu, x, w, torch.empty_like(gu), h, dx, dw, db, ctx.kind)
        dwd = torch.matmul(rows.t(), h) if need[3] else None
        return dx, dw, db, dwd, rows.sum(0) if need[4] else None, None, None


class TempoGatedFFN(nn.Module):
    """A gated feed-forward block, y = (act(g) u) down^T with [g | u] = x gate_up^T: the rows of the gate come first.  kind: "silu",
    "gelu_erf" or "gelu_tanh".  Its weights are its own parameters, drawn as nn.Linear draws them.  No second derivative."""

    def __init__(self, hidden: int, ffn: int, kind: str = "silu", bias: bool = False, dtype=torch.float32):
        super().__init__()
        if kind not in ("silu", "gelu_erf", "gelu_tanh"):
            raise ValueError(f'kind must be "silu", "gelu_erf" or "gelu_tanh", got {kind!r}')
        self.kind = kind
        for name, rows, columns in (("gate_up", 2 * ffn, hidden), ("down", hidden, ffn)):
            w = nn.Parameter(torch.empty(rows, columns, dtype=dtype))
            nn.init.kaiming_uniform_(w, a=math.sqrt(5))
            b = nn.Parameter(torch.empty(rows, dtype=dtype).uniform_(-columns ** -0.5, columns ** -0.5)) if bias else None
            self.register_parameter(name + "_weight", w)
            self.register_parameter(name + "_bias", b)

    def forward(self, x):
        args = [x, self.gate_up_weight, self.gate_up_bias, self.down_weight, self.down_bias]
        if torch.is_autocast_enabled("cuda"):    # as a Linear would take them
            args = [None if t is None else t.to(torch.get_autocast_dtype("cuda")) for t in args]
        keep = torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in args)
        with torch.autocast("cuda", enabled=False):
            return _GatedFFNFn.apply(*args, self.kind, keep)


class _EncoderLayerFn(torch.autograd.Function):
    """The whole layer, whose forward has been made (_native.tempo_encoder_fwd): keeps what the layer's parts keep for the
    inputs that require a gradient.  The backward is one native call too."""

    @staticmethod
    def forward(ctx, made, setting, store_mask, x, *params):
        qkv, probs, keep, ctxt, y1, rstd1, h, side, y2, rstd2, place = made
        wqkv, bqkv, wproj, bproj, w1, b1, w2, b2, gamma1, beta1, gamma2, beta2 = params
        # where _grads_of_parts() finds the inputs' graphs: not kept for their values, which may change
        ctx.places = place, wqkv, bqkv, wproj, bproj, w1, b1, w2, b2
        ctx.setting, ctx.store_mask = setting, store_mask
        of = ctx.needs_input_grad[3:]
        inner = of[0] or of[1] or of[2]                                        # the gradient goes on to qkv,
        first = inner or of[3] or of[4] or of[9] or of[10]                     # to the first LayerNorm,
        second = first or of[5] or of[6]                                       # to GELU
        ctx.save_for_backward(
            x if of[1] else None, wqkv if of[0] else None, wproj if inner else None, w1 if first else None,
            w2 if second else None, gamma1 if first else None, beta1 if first else None, gamma2, beta2,
            qkv if inner else None, probs if inner else None, keep if inner and store_mask else None, ctxt if of[3] else None,
            y1 if first or of[5] else None, rstd1 if first else None, h if second or of[7] else None,
            side if second else None, y2, rstd2)
        return y2

    @staticmethod
    def backward(ctx, dy):
        needed = ctx.needs_input_grad[3:]
        grads = None
        if not torch.is_grad_enabled():
            wanted = sum(1 << i for i, n in enumerate(needed) if n)
            grads = B.encoder_bwd(dy.contiguous(), wanted, *ctx.setting, *ctx.saved_tensors)
        if grads is None:     # create_graph, or a tensor that is no plain one any more: the gradients of the parts
            grads = _grads_of_parts(ctx, dy, needed)
        return (None,) * 3 + grads


class _PlaceFn(torch.autograd.Function):
    """x's place in its graph, without its values; nothing looks at those it has."""

    @staticmethod
    def forward(ctx, x):
        return x.new_empty(()).expand(x.shape)

    @staticmethod
    def backward(ctx, dx):
        return dx


class _MadeLinearFn(torch.autograd.Function):
    """y = x w^T + b, already made."""

    @staticmethod
    def forward(ctx, y, x, w, b):
        ctx.save_for_backward(x, w)
        return y.detach()

    @staticmethod
    def backward(ctx, dy):
        x, w = ctx.saved_tensors
        rows = dy.reshape(-1, dy.shape[-1])
        dx = torch.matmul(dy, w) if ctx.needs_input_grad[1] else None
        dw = torch.matmul(rows.t(), x.reshape(-1, x.shape[-1])) if ctx.needs_input_grad[2] else None
        return None, dx, dw, rows.sum(0) if ctx.needs_input_grad[3] else None


class _MadeScoresFn(torch.autograd.Function):
    """scale q k^T of every head, already made; only its place in the graph is needed."""

    @staticmethod
    def forward(ctx, scores, q, k, scale):
        ctx.scale = scale
        ctx.save_for_backward(q, k)
        return scores.detach()

    @staticmethod
    def backward(ctx, ds):
        q, k = ctx.saved_tensors
        ds = ds * ctx.scale
        return None, torch.matmul(ds, k), torch.matmul(ds.transpose(-1, -2), q), None


def _grads_of_parts(ctx, dy, needed):
    """The gradients as the layer made of its parts gives them, connected to its inputs under create_graph.  The graph of the
    parts is laid over what the forward made: nothing of the forward runs again, and only what was kept is looked at."""
    heads, ffn, p, seed, offset, kind = ctx.setting
    x, wqkv, wproj, w1, w2, g1, be1, g2, be2, qkv, probs, keep, ctxt, y1, rstd1, h, side, y2, rstd2 = ctx.saved_tensors
    Bn, S, H = dy.shape
    d = H // heads

    def value(t, *shape):     # t in that shape; zeros without memory in the place of what nothing looks at
        return dy.new_zeros(()).expand(shape) if t is None else t.reshape(shape)
    with torch.enable_grad():
        # Aliases, which are inputs of this graph alone: x may depend on these parameters, and two of them may be the same
        # tensor, whose gradients the caller's backward adds up.
        kept, places = (x, wqkv, None, wproj, None, w1, None, w2, None), ctx.places
        inputs = [t.view_as(t) if t is not None else None
                  for t in (*(p if k is None else k for k, p in zip(kept, places)), g1, be1, g2, be2)]
        x, wqkv, bqkv, wproj, bproj, w1, b1, w2, b2, g1, be1, g2, be2 = inputs

        def core(q, k, v):
            scores = _MadeScoresFn.apply(value(None, Bn, heads, S, S), q, k, 1.0 / math.sqrt(d))
            made = (probs, keep, value(ctxt, Bn, S, heads, d).permute(0, 2, 1, 3))
            return _AttentionCoreFn.apply(scores, v, None, False, p, seed, offset, ctx.store_mask, made)

        rows = value(None, Bn, S, H)
        x, g1, be1 = (value(t, *shape) for t, shape in ((x, (Bn, S, H)), (g1, (H,)), (be1, (H,))))
        a = _attention(_MadeLinearFn.apply(value(qkv, Bn, S, 3 * H), x, wqkv, bqkv), dy.shape, heads, core)
        y1 = _InplaceLayerNormFn.apply(x + _MadeLinearFn.apply(rows, a, wproj, bproj), g1, be1, None,
                                       (value(y1, Bn, S, H), rstd1))
        h = _InplaceGELUFn.apply(_MadeLinearFn.apply(value(None, Bn, S, ffn), y1, w1, b1), kind, (value(h, Bn, S, ffn), side))
        out = _InplaceLayerNormFn.apply(y1 + _MadeLinearFn.apply(rows, h, w2, b2), g2, be2, None, (y2, rstd2))
    grads = iter(torch.autograd.grad(out, [t for t, n in zip(inputs, needed) if n], dy, create_graph=torch.is_grad_enabled()))
    return tuple(next(grads) if n else None for n in needed)


def _attention(qkv, shape, heads, core):
    Bn, S, H = shape
    q, k, v = qkv.view(Bn, S, 3, heads, H // heads).permute(2, 0, 3, 1, 4)
    return core(q, k, v.contiguous()).permute(0, 2, 1, 3).reshape(Bn, S, H)


class TempoEncoderLayer(nn.Module):
    """A post-LN BERT encoder layer built from the three memory-reduced layers (Fig. 1 of the
    paper); hidden-state dropouts are left out (they are not part of the method).  rotary: a RotaryPositions that q and k go
    through; gated: the kind of a TempoGatedFFN in the place of the two feed-forward layers and GELU."""

    def __init__(self, hidden: int, heads: int, ffn: int, p_attn: float = 0.1, eps: float = 1e-12,
                 dtype=torch.float32, rotary: Optional[RotaryPositions] = None, gated: Optional[str] = None):
        super().__init__()
        self.heads = heads
        self.qkv = nn.Linear(hidden, 3 * hidden, dtype=dtype)
        self.proj = nn.Linear(hidden, hidden, dtype=dtype)
        if gated is None:
            self.fc1 = nn.Linear(hidden, ffn, dtype=dtype)
            self.fc2 = nn.Linear(ffn, hidden, dtype=dtype)
        else:
            self.ffn = TempoGatedFFN(hidden, ffn, gated, True, dtype)
        self.ln1 = InplaceLayerNorm(hidden, eps)
        self.ln2 = InplaceLayerNorm(hidden, eps)
        if gated is None:
            self.act = InplaceGELU()
        self.core = TempoAttentionCore(p_attn)
        if rotary is not None:
            self.rotary = rotary

    def forward(self, x, key_len=None, positions=None):
        rotary = self._modules.get("rotary")
        if positions is not None and rotary is None:
            raise ValueError("positions are those of rotary, which this layer has none of")
        out = self._as_one(x, key_len) if rotary is None else None
        if out is not None:
            return out

        def core(q, k, v):
            if rotary is not None:
                q, k = rotary(q, k, positions)
            scores = torch.matmul(q, k.transpose(-1, -2)) * (1.0 / math.sqrt(q.shape[-1]))
            return self.core(scores, v, key_len)
        Bn, S, H = x.shape
        ctxt = _attention(self.qkv(x), (Bn, S, H), self.heads, core)
        x = self.ln1(x + self.proj(ctxt))
        ffn = self._modules.get("ffn")
        return self.ln2(x + (self.fc2(self.act(self.fc1(x))) if ffn is None else ffn(x)))

    def _as_one(self, x, key_len):
        """The layer as one native call each way, or None where something may see or change its parts: hooks, other
        modules in their places, a forward, a call or a product replaced, autocast, function transforms, tracing, dispatch
        and function modes, forward-mode AD, tensor subclasses, other types and layouts."""
        if torch.compiler.is_compiling():
            return None
        if not _plain(x):
            return None
        if (torch.is_autocast_enabled() or torch._C._len_torch_dispatch_stack() or torch._C._len_torch_function_stack()
                or torch._C._functorch.peek_interpreter_stack() is not None or forward_ad._current_level >= 0
                or torch.jit.is_tracing() or module._has_any_global_hook() or _calls() != _CALLS):
            return None
        parts = self._modules
        for name, kind in _PARTS:
            m = parts.get(name)
            if (type(m) is not kind or m._forward_hooks or m._forward_pre_hooks or m._backward_hooks
                    or m._backward_pre_hooks or "forward" in m.__dict__ or m._compiled_call_impl is not None):
                return None
        qkv, proj, fc1, fc2, ln1, ln2, core = (parts[n] for n in ("qkv", "proj", "fc1", "fc2", "ln1", "ln2", "core"))
        params = (qkv.weight, qkv.bias, proj.weight, proj.bias, fc1.weight, fc1.bias, fc2.weight, fc2.bias,
                  ln1.weight, ln1.bias, ln2.weight, ln2.bias)
        p, kind = core.p if core.training else 0.0, parts["act"].kind
        made = B.encoder_fwd(x, key_len, core.__dict__, self.heads, ln1.eps, ln2.eps, p, core.seed, kind, *params)
        if made is None:
            return None
        offset, *made = made
        if not torch.is_grad_enabled():
            return made[8]
        setting = (self.heads, fc1.weight.shape[0], p, core.seed, offset, kind)
        made.append(_PlaceFn.apply(x) if x.requires_grad and not qkv.weight.requires_grad else None)    # else x itself is kept
        return _EncoderLayerFn.apply(made, setting, core.store_mask, x, *params)


def _plain(x):
    if type(x) not in (torch.Tensor, nn.Parameter) or x.dtype != torch.float32 or not x.is_cuda:
        return False
    B.load()
    return B._native is not None


_PARTS = (("qkv", nn.Linear), ("proj", nn.Linear), ("fc1", nn.Linear), ("fc2", nn.Linear), ("ln1", InplaceLayerNorm),
          ("ln2", InplaceLayerNorm), ("act", InplaceGELU), ("core", TempoAttentionCore))


def _calls():
    """What a layer made of its parts goes through."""
    return (nn.Linear.forward, InplaceLayerNorm.forward, InplaceGELU.forward, TempoAttentionCore.forward, nn.Linear.__call__,
            InplaceLayerNorm.__call__, InplaceGELU.__call__, TempoAttentionCore.__call__, F.linear, torch.matmul)


_CALLS = _calls()                                # what the native call stands for
if _CALLS[0].__globals__ is not vars(linear) or _CALLS[4] is not nn.Module._wrapped_call_impl or F.linear is not torch._C._nn.linear:
    _CALLS = None                                # replaced before this module was loaded
