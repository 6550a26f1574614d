"""LLaMA-style decoder block around the library's linear layer: integration and timing harness.

The seven linear layers (q, k, v, o, gate, up, down) run through the C-ABI calls, wired into
torch autograd by a ``torch.autograd.Function`` whose backward issues the adapter backward, the
input gradient with the doubly pruned weight and the masked compressed weight gradient
(Eq. (sparse_forward), Eq. (sparse_backward_input), Eq. (sparse_backward_weight), Eq. (concat)).
Everything between them -- RMS normalisation without gain, causal attention without positional
rotation, the SiLU gate, the residual adds -- is by default plain torch in bf16 and is then NOT part of the
library: it is there so that the linears see a real data flow, each one fed by the previous
one's output and its gradient by the next one's.  ``DenseLinear`` is the same block on
``torch.nn.functional.linear`` (cuBLAS) for the all-dense comparison.

With ``norms`` the block has the layer norms of GPT-2, OPT and BERT instead, on the library's calls, residual adds
included (``LayerNorm``).  ``checkpoint=True`` of a layer keeps what its backward pass needs of its input in 8 bits: the layer norm of the
stream, the linears of their inputs; linears that share an input share its checkpoint, which the layer norm in front of them writes.
Their calls' workspaces (a decoded matrix of activations among them) are allocated for the one call and go back to torch's caching
allocator behind it, so that all layers of a model use the same memory in turn and nothing stays; what a captured graph needs comes from
that graph's own pool.

With ``attention`` queries and keys are turned by their positions and attention runs on the library's calls (``Attention``): shared key
heads, windows, packed and padded batches.

Every linear call is bracketed by CUDA events when ``timers`` is given, so the time spent in
the linears can be summed separately from the torch glue.
"""
from __future__ import annotations

from typing import Dict, List, Optional, Tuple

import torch
import torch.nn.functional as F
from torch.autograd.function import once_differentiable

from . import binding as B

LAYER_NAMES = ("q", "k", "v", "o", "gate", "up", "down")
Timers = List[Tuple[torch.cuda.Event, torch.cuda.Event]]


def _timed(timers: Optional[Timers], fn):
    if timers is None:
        return fn()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    out = fn()
    e1.record()
    timers.append((e0, e1))
    return out


def elapsed_ms(timers: Timers) -> float:
    """Sum of the bracketed intervals; synchronise the device first."""
    return sum(a.elapsed_time(b) for a, b in timers)


class SlopeLinear:
    """One 2:4-sparse layer: compressed weight and its doubly pruned transposed copy, static masks,
    optional lazy adapters, and the gradient buffers the backward fills (dWc compressed, dL, dR)."""

    def __init__(self, W: torch.Tensor, L: Optional[torch.Tensor] = None, R: Optional[torch.Tensor] = None,
                 max_tokens: int = 0, checkpoint: bool = False):
        self.d_out, self.d_in = W.shape
        self.Wc_vals, self.Wc_meta, self.mask1 = B.alloc_compressed(self.d_out, self.d_in)
        self.WTc_vals, self.WTc_meta, _ = B.alloc_compressed(self.d_in, self.d_out)
        B.slope_prune_24_double(W, self.Wc_vals, self.Wc_meta, self.mask1, self.WTc_vals, self.WTc_meta, None)
        self.L, self.R = L, R
        self.r = 0 if L is None else L.shape[1]
        self.dWc = torch.empty_like(self.Wc_vals)
        self.dL = None if L is None else torch.empty_like(L)
        self.dR = None if R is None else torch.empty_like(R)
        self.workspace = None
        if self.r and max_tokens and not checkpoint:
            n = B.slope_adapter_workspace_bytes(max_tokens, self.d_out, self.d_in, self.r)
            self.workspace = torch.empty(max(n, 16), dtype=torch.uint8, device=W.device)
        self.checkpoint = checkpoint
        self.timers: Optional[Timers] = None

    def __call__(self, X: torch.Tensor, kept: Optional[torch.Tensor] = None) -> torch.Tensor:
        """``kept``: a checkpoint of X that is there already (``checkpoint`` layers; else they store one)."""
        return _SlopeLinearFn.apply(X, self, kept)


def _scratch(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(nbytes, 16), dtype=torch.uint8, device=device)


class _SlopeLinearFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, layer: SlopeLinear, kept):
        X = X.contiguous()
        b = X.shape[0]
        Y = torch.empty(b, layer.d_out, dtype=torch.bfloat16, device=X.device)
        T = None

        def run():
            nonlocal T, kept
            if layer.r:
                T = torch.empty(b, layer.r, dtype=torch.bfloat16, device=X.device)
                B.slope_linear_fwd_adapter(X, layer.Wc_vals, layer.Wc_meta, layer.d_out, layer.L, layer.R, T, Y)
            else:
                B.slope_linear_fwd(X, layer.Wc_vals, layer.Wc_meta, layer.d_out, Y)
            if layer.checkpoint and kept is None:
                kept = B.alloc_checkpoint(b, layer.d_in, X.device)
                B.slope_checkpoint_store(X, kept)

        _timed(layer.timers, run)
        ctx.layer = layer
        saved = kept if layer.checkpoint else X
        ctx.save_for_backward(saved, T) if T is not None else ctx.save_for_backward(saved)
        return Y

    @staticmethod
    @once_differentiable                 # (linear in dY: with a dY that is a constant there is nothing to refuse)
    def backward(ctx, dY):
        layer: SlopeLinear = ctx.layer
        saved = ctx.saved_tensors
        X, T = saved[0], (saved[1] if len(saved) > 1 else None)
        dY = dY.contiguous()
        b = dY.shape[0]
        dX = torch.empty(b, layer.d_in, dtype=torch.bfloat16, device=dY.device)
        sizes = (b, layer.d_out, layer.d_in, layer.r)

        def run():
            dT = None
            if layer.r:
                dT = torch.empty(b, layer.r, dtype=torch.bfloat16, device=dY.device)
                if layer.checkpoint:
                    B.slope_adapter_fwd_bwd(2, None, dY, None, layer.R, *sizes, dT=dT)
                else:
                    need = B.slope_adapter_workspace_bytes(*sizes)
                    if layer.workspace is None or layer.workspace.numel() < need:
                        layer.workspace = _scratch(need, dY.device)
                    B.slope_adapter_fwd_bwd(1, X, dY, layer.L, layer.R, *sizes, T=T, dT=dT, dL=layer.dL, dR=layer.dR, workspace=layer.workspace)
            B.slope_linear_bwd_dx(dY, layer.WTc_vals, layer.WTc_meta, layer.d_in, dX, dT, layer.L)
            if not layer.checkpoint:
                B.slope_linear_bwd_dw_masked(dY, X, layer.mask1, layer.dWc)
                return
            workspace = _scratch(B.slope_bwd_dw_q8_workspace_bytes(*sizes), dY.device)
            if layer.r:
                B.slope_linear_bwd_dw_adapter_q8(dY, X, T, dT, layer.mask1, layer.dWc, layer.dL, layer.dR, workspace)
            else:
                B.slope_linear_bwd_dw_masked_q8(dY, X, layer.mask1, layer.dWc, workspace)

        _timed(layer.timers, run)
        return dX, None, None


class _FirstDerivativeFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, gradient, of):
        ctx.of = of
        return gradient.view_as(gradient)

    @staticmethod
    def backward(ctx, _):
        raise RuntimeError(f"{ctx.of} has no second derivative")


def _first_derivative(gradient: torch.Tensor, of: str) -> torch.Tensor:
    """A gradient that depends on inputs as well as on the gradient that came in: where a graph of the backward pass is asked for, going back
    through it is an error, instead of a derivative that lacks this part."""
    return _FirstDerivativeFn.apply(gradient.requires_grad_(True), of) if torch.is_grad_enabled() else gradient


class LayerNorm:
    """Layer norm over the library's calls, with the residual addition in front of it: gain and offset, and the gradient buffers that the
    backward fills (dgamma, dbeta).  ``checkpoint``: the stream is kept in 8 bits for the backward pass, and so is the output for
    the linears behind."""

    def __init__(self, gamma: torch.Tensor, beta: torch.Tensor, eps: float = 1e-5, checkpoint: bool = False):
        self.gamma, self.beta, self.eps, self.checkpoint = gamma, beta, eps, checkpoint
        self.dgamma, self.dbeta = torch.empty_like(gamma), torch.empty_like(beta)

    def __call__(self, X: torch.Tensor, residual: Optional[torch.Tensor] = None):
        """(stream, output, checkpoint of the output or None): the stream is X, or X + residual."""
        return _LayerNormFn.apply(X, residual, self)


class _LayerNormFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, residual, norm: LayerNorm):
        X = X.contiguous()
        residual = None if residual is None else residual.contiguous()
        b, d = X.shape
        Y = torch.empty(b, d, dtype=torch.bfloat16, device=X.device)
        H = None if residual is None else torch.empty_like(X)
        mean, rstd = (torch.empty(b, dtype=torch.float32, device=X.device) for _ in range(2))
        H_ckpt, Y_ckpt = (B.alloc_checkpoint(b, d, X.device) for _ in range(2)) if norm.checkpoint else (None, None)
        B.slope_layer_norm_fwd(X, norm.gamma, norm.beta, norm.eps, Y, mean, rstd, residual, H, H_ckpt, Y_ckpt)
        ctx.norm, ctx.dtype, ctx.with_residual = norm, X.dtype, residual is not None
        ctx.save_for_backward(H_ckpt if norm.checkpoint else X if H is None else H, mean, rstd)
        ctx.set_materialize_grads(False)
        if Y_ckpt is not None:
            ctx.mark_non_differentiable(Y_ckpt)
        return X.view_as(X) if H is None else H, Y, Y_ckpt

    @staticmethod
    def backward(ctx, dH, dY, _):
        norm: LayerNorm = ctx.norm
        if dY is None:                       # only the stream was used
            norm.dgamma.zero_()
            norm.dbeta.zero_()
            return dH, dH if ctx.with_residual else None, None
        H, mean, rstd = ctx.saved_tensors
        dY = dY.contiguous()
        b, d = dY.shape
        dX = torch.empty(b, d, dtype=ctx.dtype, device=dY.device)
        workspace = _scratch(B.slope_layer_norm_bwd_workspace_bytes(b, d), dY.device)
        B.slope_layer_norm_bwd(dY, H, mean, rstd, norm.gamma, dX, norm.dgamma, norm.dbeta, workspace, None if dH is None else dH.contiguous())
        dX = _first_derivative(dX, "LayerNorm")
        # (the residual is a sub-layer's bf16 output, whatever the stream's type)
        return dX, dX.to(torch.bfloat16) if ctx.with_residual else None, None


class Attention:
    """Softmax attention over the library's calls, behind the rotation of queries and keys by their positions if there are ``frequencies``
    (``binding.rotary_frequencies``).  A call takes the three projections' outputs [tokens x heads * head_dim] and says where the sequences lie;
    ``positions`` int32 [tokens].  Rows of no sequence have an output and gradients of zero.  The backward pass is over the same sequences and
    positions: these tensors and the frequencies must not be written in place before it (an error, as for any tensor that autograd keeps)."""

    def __init__(self, heads: int, kv_heads: Optional[int] = None, frequencies: Optional[torch.Tensor] = None, factor: float = 1.0,
                 interleaved: bool = False, causal: bool = True, window: int = 0, scale: Optional[float] = None):
        self.heads, self.kv_heads = heads, heads if kv_heads is None else kv_heads
        self.frequencies, self.factor, self.interleaved = frequencies, factor, interleaved
        self.mask = {"causal": causal, "window": window, "scale": scale}

    def __call__(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, sequences: Optional[int] = None, starts: Optional[torch.Tensor] = None,
                 lengths: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None) -> torch.Tensor:
        if (self.frequencies is None) != (positions is None):
            raise ValueError("Attention: positions and frequencies belong together")
        return _AttentionFn.apply(q, k, v, self, {"sequences": sequences, "starts": starts, "lengths": lengths, **self.mask}, positions)


class _AttentionFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, layer: Attention, batch, positions):
        b, head_dim = q.shape[0], q.shape[1] // layer.heads
        if q.shape[1] % layer.heads or k.shape[1] != layer.kv_heads * head_dim:
            raise ValueError("Attention: the projections do not have these heads")
        # (what the layer says now is what the backward pass goes by: another table, factor or mask is for the calls that follow)
        frequencies, turn = layer.frequencies, {"factor": layer.factor, "interleaved": layer.interleaved}
        if positions is not None:
            turned = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty_like(k, memory_format=torch.contiguous_format)
            B.slope_rotary(q, k, positions, frequencies, head_dim, *turned, **turn)
            q, k = turned
        # (rows of no sequence are not written)
        ctx.fresh = torch.empty if batch["starts"] is None and batch["lengths"] is None else torch.zeros
        O = ctx.fresh(b, layer.heads * head_dim, dtype=q.dtype, device=q.device)
        lse = torch.empty(layer.heads, b, dtype=torch.float32, device=q.device)
        B.slope_attention_fwd(q, k, v, head_dim, O, lse, **batch)
        starts, lengths = batch.pop("starts"), batch.pop("lengths")
        ctx.batch, ctx.turn, ctx.sizes = batch, turn, (b, layer.heads, layer.kv_heads, head_dim)
        # (where the sequences lie and the positions, too: one that is written before the backward pass is an error there, not other gradients)
        # (autograd keeps no tensor of inference mode: a table that was made in it, as evaluation does, goes in as a copy)
        kept = (t.clone() if t is not None and t.is_inference() else t for t in (starts, lengths, positions, frequencies))
        ctx.save_for_backward(q, k, v, O, lse, *kept)
        return O

    @staticmethod
    def backward(ctx, dO):
        q, k, v, O, lse, starts, lengths, positions, frequencies = ctx.saved_tensors
        head_dim = ctx.sizes[3]
        grads = [ctx.fresh(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v)]
        workspace = _scratch(B.slope_attention_bwd_workspace_bytes(*ctx.sizes), q.device)
        B.slope_attention_bwd(dO.contiguous(), q, k, v, O, lse, head_dim, *grads, workspace, starts=starts, lengths=lengths, **ctx.batch)
        if positions is not None:
            dq, dk = grads[:2]
            B.slope_rotary(dq, dk, positions, frequencies, head_dim, dq, dk, **ctx.turn, backward=True)
        return (*(_first_derivative(g, "Attention") for g in grads), None, None, None)


class DenseLinear:
    """The dense bf16 layer on torch (cuBLAS): Y = X W^T, gradients by autograd."""

    def __init__(self, W: torch.Tensor):
        self.W = W.clone().requires_grad_(True)
        self.timers: Optional[Timers] = None

    def __call__(self, X: torch.Tensor, kept: Optional[torch.Tensor] = None) -> torch.Tensor:
        return _DenseLinearFn.apply(X, self.W, self)


class _DenseLinearFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, W, layer: DenseLinear):
        ctx.layer = layer
        ctx.save_for_backward(X, W)
        return _timed(layer.timers, lambda: F.linear(X, W))

    @staticmethod
    def backward(ctx, dY):
        X, W = ctx.saved_tensors
        dX, dW = _timed(ctx.layer.timers, lambda: (dY @ W, dY.t() @ X))
        return dX, dW, None


def rms_norm(x: torch.Tensor, eps: float) -> torch.Tensor:
    xf = x.float()
    return (xf * torch.rsqrt((xf * xf).mean(dim=-1, keepdim=True) + eps)).to(x.dtype)


def causal_attention(q, k, v, batch: int, seq: int, heads: int) -> torch.Tensor:
    hd = q.shape[1] // heads
    split = lambda t: t.reshape(batch, seq, heads, hd).permute(0, 2, 1, 3)
    out = F.scaled_dot_product_attention(split(q), split(k), split(v), is_causal=True)
    return out.permute(0, 2, 1, 3).reshape(batch * seq, heads * hd)


def decoder_block(x: torch.Tensor, layers: Dict[str, object], batch: int, seq: int, heads: int,
                  eps: float = 1e-5, norms: Optional[Dict[str, LayerNorm]] = None, attention: Optional[Attention] = None,
                  positions: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [batch*seq, d] bf16 -> block output [batch*seq, d] bf16; ``layers`` maps the seven names to callables, ``norms`` "attention"
    and "mlp" to layer norms (None: RMS normalisation in torch).  ``attention`` with its ``positions`` takes the place of torch's."""
    if attention is None:
        attend = lambda q, k, v: causal_attention(q, k, v, batch, seq, heads)
    else:
        attend = lambda q, k, v: attention(q, k, v, sequences=batch, positions=positions)
    if norms is None:
        n1 = rms_norm(x, eps)
        a = attend(layers["q"](n1), layers["k"](n1), layers["v"](n1))
        h = x + layers["o"](a)
        n2 = rms_norm(h, eps)
        g = F.silu(layers["gate"](n2)) * layers["up"](n2)
        return h + layers["down"](g)
    x, n1, kept = norms["attention"](x)
    a = attend(layers["q"](n1, kept), layers["k"](n1, kept), layers["v"](n1, kept))
    h, n2, kept = norms["mlp"](x, layers["o"](a))
    g = F.silu(layers["gate"](n2, kept)) * layers["up"](n2, kept)
    return h + layers["down"](g)


def block_step(x: torch.Tensor, dout: torch.Tensor, layers: Dict[str, object], batch: int, seq: int, heads: int,
               eps: float = 1e-5, norms: Optional[Dict[str, LayerNorm]] = None, attention: Optional[Attention] = None,
               positions: Optional[torch.Tensor] = None):
    """One training step of the block for the loss <out, dOut> (no optimizer): returns (out, dx)."""
    x = x.detach().requires_grad_(True)
    out = decoder_block(x, layers, batch, seq, heads, eps, norms, attention, positions)
    out.backward(dout)
    return out.detach(), x.grad
