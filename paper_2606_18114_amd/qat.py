"""Quantization-aware training with the ternary linear layer (paper Sec. 3.1).

``TernaryLinear`` replaces a Mamba-2 ``in_proj`` / ``out_proj``: it keeps
float32 latent weights, and on every forward call

  * recomputes the group scales and ternary codes from the current weights
    (``tm_ternarize_pack``; the scale is not a learned parameter),
  * applies the dequantized weights to the bfloat16 activations
    (``tm_tgemm_fwd``, float32 output);

and its backward pass is the straight-through estimator: the gradient passes
the quantizer unchanged, so ``dX = dY . (q s)`` (``tm_tgemm_bwd_dx_f16``:
one float16 pass, each dequantized weight within 2^-11 relative; or the
two-pass ``tm_tgemm_bwd_dx`` with ``dx_precision="exact"``) and
``dW = dY^T . X`` (``tm_tgemm_bwd_dw_ste``).  The incoming gradient is taken
in bfloat16, the precision the backward kernels read.

The scale variants the paper tests against this layer are options of the
same module: a learned magnitude next to the absmean threshold (decoupled),
a learned scale that is threshold and magnitude at once (learnable, whose
zero ratio collapses in Sec. 4), and per-row threshold multipliers (the
appendix's 0.8 x absmean on the gate rows).  Their extra calls are
``tm_ternarize_pack_thresh``, ``tm_ternarize_codes`` and, in the backward,
``tm_group_code_dot`` for the gradient of the learned scale.

Every product runs in the library's kernels; this module only wires them
into autograd (a dtype cast of the gradient and reshapes are the only torch
operations on the data).  ``pack_for_decode`` returns the deployment format
(2-bit codes and float16 group scales) that ``ops.tgemv`` reads.

``Mamba2Mixer`` is the unquantized part between the two projections over whole
sequences, ``Embedding`` the residual stream's beginning; with ``TernaryLinear``
they make up a block's training step on the library's kernels.
"""

from __future__ import annotations

import math
from typing import Optional, Tuple

import torch
from torch.autograd.function import once_differentiable

from . import ops


SCALE_MODES = ("absmean", "decoupled", "learnable", "learnable_ste")


class TernaryLinearFn(torch.autograd.Function):
    """y = x . (q m)^T with straight-through backward.

    mode "absmean": q and the magnitude m = s are recomputed from `weight`
    (Sec. 3.1); `scale` is None.  mode "decoupled": q from the recomputed
    absmean threshold, m = `scale` (a learned alpha_g, appendix Decoupled
    Quantization Ablations).  mode "learnable": `scale` is the learned s_g of
    Sec. 4, used as the rounding threshold and as the magnitude.  `row_mult`
    (float32 [out] or None) multiplies each row's absmean threshold.
    In "decoupled" and "learnable" the gradient of the learned scale is
    sum_group q * dWhat (the hard forward rounding passes nothing back
    through the threshold) and the weights get dWhat.  "learnable_ste" has
    the same forward as "learnable", with only the rounding straight-through:
    the scale also receives the threshold term, and the weights' gradient is
    clip-masked (``tm_scale_ste_grad``).
    """

    @staticmethod
    def forward(ctx, x: torch.Tensor, weight: torch.Tensor, scale: Optional[torch.Tensor],
                g: int, eps: float, zero_count: Optional[torch.Tensor], mode: str,
                row_mult: Optional[torch.Tensor],
                out_dtype: torch.dtype = torch.float32,
                dx_precision: str = "f16") -> torch.Tensor:
        N, K = weight.shape
        if x.shape[-1] != K:
            raise ValueError(f"x has {x.shape[-1]} features, the layer takes {K}")
        lead = x.shape[:-1]
        x2 = x.reshape(-1, K)
        if x2.dtype != torch.bfloat16:
            raise TypeError(f"x must be bfloat16 (got {x2.dtype}): the layer is W1.58A16")
        x2 = x2.contiguous()
        w = weight.detach().contiguous()
        want_zc = zero_count is not None
        if mode in ("learnable", "learnable_ste"):
            mag = scale.detach().contiguous()
            codes, _ = ops.ternarize_codes(w, mag, g, eps, zero_count=zero_count,
                                           want_zero_count=want_zc)
        else:
            codes, absmean, _, _ = ops.ternarize_pack(w, g, eps, zero_count=zero_count,
                                                      want_f16=False, want_zero_count=want_zc,
                                                      row_mult=row_mult)
            mag = absmean if mode == "absmean" else scale.detach().contiguous()
        y = ops.tgemm_fwd(x2, codes, mag, g, out_dtype=out_dtype)
        ctx.save_for_backward(x2, codes, mag, w if mode == "learnable_ste" else None)
        ctx.g = g
        ctx.eps = eps
        ctx.ste_scale = mode == "learnable_ste"
        ctx.lead = lead
        ctx.x_dtype = x.dtype
        ctx.learned = mode != "absmean"
        ctx.dx_precision = dx_precision
        return y.reshape(*lead, N)

    @staticmethod
    def backward(ctx, gy: torch.Tensor):
        x2, codes, mag, w = ctx.saved_tensors
        N = codes.shape[0]
        dy = gy.reshape(-1, N)
        dx = dw = dscale = None
        if ctx.needs_input_grad[0]:
            # rounds a contiguous float32 gradient to bfloat16 on the way, and dX once
            if not (dy.dtype == torch.float32 and dy.is_contiguous()):
                dy = dy.to(torch.bfloat16)
            dx, dy = ops.layer_input_grad(dy.contiguous(), codes, mag, ctx.g,
                                          precision=ctx.dx_precision)
            dx = dx.to(ctx.x_dtype).reshape(*ctx.lead, x2.shape[1])
        else:
            if dy.dtype != torch.bfloat16:
                dy = dy.to(torch.bfloat16)
            dy = dy.contiguous()
        want_scale = ctx.learned and ctx.needs_input_grad[2]
        if ctx.needs_input_grad[1] or want_scale:
            dw_hat = ops.tgemm_bwd_dw_ste(dy, x2)   # gradient w.r.t. the dequantized weights
            if ctx.ste_scale:
                # scale gradient with the threshold term; the weights' gradient
                # clip-masked, written over dWhat
                dscale, dw_m = ops.scale_ste_grad(w, codes, mag, dw_hat, ctx.g, ctx.eps,
                                                  in_place=ctx.needs_input_grad[1],
                                                  want_dW=ctx.needs_input_grad[1])
                if ctx.needs_input_grad[1]:
                    dw = dw_m
                if not want_scale:
                    dscale = None
            else:
                if want_scale:
                    dscale = ops.group_code_dot(codes, dw_hat, ctx.g)
                if ctx.needs_input_grad[1]:
                    dw = dw_hat
        return dx, dw, dscale, None, None, None, None, None, None, None


class TernaryLinear(torch.nn.Module):
    """Grouped-absmean ternary linear layer (no bias; the Mamba-2 projections
    have none).  weight: float32 [out_features, in_features]; groups of `g`
    consecutive input features of one output row share a scale.

    scale_mode "absmean" (the paper's layer): the scale is recomputed from
    the weights on every call and is not a parameter.  "decoupled": codes
    from the recomputed absmean, magnitude the parameter `scale`.
    "learnable": the parameter `scale` is both threshold and magnitude;
    "learnable_ste": the same with only the rounding straight-through (the
    scale's gradient keeps the threshold term, the weights' is clip-masked).
    The parameter starts at the absmean of the weights (``reset_scale``, run on
    the first call unless it was run before or the scale was loaded with
    ``load_state_dict``).  threshold_mult (float32 [out]) scales
    each row's absmean threshold (e.g. 0.8 on the gate rows of in_proj).
    out_dtype: float32 (default) or bfloat16, the output rounded once as a
    bfloat16 model stores it; the incoming gradient then needs no cast.
    dx_precision: "f16" (default, one float16 pass for the input gradient)
    or "exact" (two bfloat16 passes, 16 bits of every scale).
    """

    def __init__(self, in_features: int, out_features: int, g: int = 128, eps: float = 1e-5,
                 device: Optional[torch.device] = None, track_zero_ratio: bool = True,
                 scale_mode: str = "absmean", threshold_mult: Optional[torch.Tensor] = None,
                 out_dtype: torch.dtype = torch.float32, dx_precision: str = "f16"):
        super().__init__()
        if dx_precision not in ("f16", "exact"):
            raise ValueError("dx_precision must be 'f16' or 'exact'")
        self.dx_precision = dx_precision
        if out_dtype not in (torch.float32, torch.bfloat16):
            raise ValueError("out_dtype must be torch.float32 or torch.bfloat16")
        self.out_dtype = out_dtype
        if in_features % g or in_features % 64:
            raise ValueError(f"in_features={in_features} must be a multiple of g={g} and of 64")
        if scale_mode not in SCALE_MODES:
            raise ValueError(f"scale_mode must be one of {SCALE_MODES}")
        if threshold_mult is not None:
            if scale_mode in ("learnable", "learnable_ste"):
                raise ValueError("a learnable scale is its own threshold: no threshold_mult")
            if threshold_mult.shape != (out_features,):
                raise ValueError(f"threshold_mult must have shape ({out_features},)")
        self.in_features, self.out_features, self.g, self.eps = in_features, out_features, g, eps
        self.scale_mode = scale_mode
        self.weight = torch.nn.Parameter(
            torch.empty((out_features, in_features), dtype=torch.float32, device=device))
        torch.nn.init.normal_(self.weight, 0.0, 0.02)
        if scale_mode == "absmean":
            self.scale = None
        else:
            self.scale = torch.nn.Parameter(
                torch.zeros((out_features, in_features // g), dtype=torch.float32, device=device))
        self._scale_ready = scale_mode == "absmean"
        # a scale that arrives through load_state_dict (a checkpoint, a resumed
        # run) is the trained one: it must not be reset to the absmean
        self.register_load_state_dict_pre_hook(TernaryLinear._mark_scale_loaded)
        self.register_buffer(
            "threshold_mult",
            None if threshold_mult is None
            else threshold_mult.detach().to(device=device, dtype=torch.float32).contiguous())
        self._zc = (torch.zeros((1,), dtype=torch.int64, device=device)
                    if track_zero_ratio else None)

    @classmethod
    def from_weight(cls, weight: torch.Tensor, g: int = 128, eps: float = 1e-5,
                    **kw) -> "TernaryLinear":
        """Wrap existing (e.g. pretrained) float weights [out, in]."""
        m = cls(weight.shape[1], weight.shape[0], g, eps, device=weight.device, **kw)
        with torch.no_grad():
            m.weight.copy_(weight.float())
        if m.scale is not None and weight.is_cuda:
            m.reset_scale()
        return m

    @staticmethod
    def _mark_scale_loaded(module, state_dict, prefix, *args) -> None:
        if module.scale is not None and (prefix + "scale") in state_dict:
            module._scale_ready = True

    @torch.no_grad()
    def reset_scale(self) -> None:
        """Set the learned scale to the absmean of the current weights."""
        if self.scale is None:
            raise RuntimeError("the absmean layer has no scale parameter")
        ops.ternarize_pack(self.weight.detach().contiguous(), self.g, self.eps,
                           scales=self.scale.data, want_f16=False, want_zero_count=False)
        self._scale_ready = True

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        if self._zc is not None and self._zc.device != self.weight.device:
            self._zc = self._zc.to(self.weight.device)
        if not self._scale_ready:
            self.reset_scale()
        return TernaryLinearFn.apply(x, self.weight, self.scale, self.g, self.eps, self._zc,
                                     self.scale_mode, self.threshold_mult, self.out_dtype,
                                     self.dx_precision)

    def zero_ratio(self) -> float:
        """Fraction of zero codes in the last forward call (Sec. 3.1 tracks it
        during training); reading it synchronizes with the device."""
        if self._zc is None:
            raise RuntimeError("zero-ratio tracking is off for this layer")
        return int(self._zc.item()) / (self.in_features * self.out_features)

    @torch.no_grad()
    def pack_for_decode(self) -> Tuple[torch.Tensor, torch.Tensor]:
        """(codes uint8 [out, in/4], scales float16 [out, in/g]) of the current
        weights: the storage format of the decode GEMV."""
        w = self.weight.detach().contiguous()
        if self.scale_mode == "absmean":
            codes, _, s16, _ = ops.ternarize_pack(w, self.g, self.eps, want_zero_count=False,
                                                  row_mult=self.threshold_mult)
            return codes, s16
        if self.scale_mode in ("learnable", "learnable_ste"):
            codes, _ = ops.ternarize_codes(w, self.scale.detach().contiguous(), self.g, self.eps,
                                           want_zero_count=False)
        else:
            codes, _, _, _ = ops.ternarize_pack(w, self.g, self.eps, want_f16=False,
                                                want_zero_count=False,
                                                row_mult=self.threshold_mult)
        return codes, self.scale.detach().to(torch.float16)

    def extra_repr(self) -> str:
        return (f"in_features={self.in_features}, out_features={self.out_features}, "
                f"g={self.g}, eps={self.eps}, scale_mode={self.scale_mode}, "
                f"out_dtype={self.out_dtype}")


class Mamba2MixerFn(torch.autograd.Function):
    """The mixer between the projections over packed sequences: convolution,
    selective scan, gated norm (``tm_mixer_conv``, ``_scan``, ``_norm``) and
    their gradients.  zxbcdt [T, Z]; offsets int32 [nseq + 1] or None.  whole:
    the sequences cover every row."""

    @staticmethod
    def forward(ctx, zx, conv_w, conv_b, dt_bias, A_log, D, norm_w, offsets, eps, whole):
        new = torch.empty if whole else torch.zeros
        out = new((zx.shape[0], norm_w.shape[0]), dtype=torch.bfloat16, device=zx.device)
        par = [p.detach().contiguous() for p in (conv_w, conv_b, dt_bias, A_log, D, norm_w)]
        zx = zx.contiguous()
        u = ops.mixer_conv(zx, par[0], par[1], offsets)
        y = ops.mixer_scan(u, zx, *par[2:5], offsets)
        ops.mixer_norm(y, zx, par[5], eps, out, offsets)
        ctx.save_for_backward(zx, u, y, offsets, *par)
        ctx.eps, ctx.whole = eps, whole
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        zx, u, y, offsets, conv_w, conv_b, dt_bias, A_log, D, norm_w = ctx.saved_tensors
        dout = dout.to(torch.bfloat16).contiguous()
        dzx = torch.empty_like(zx) if ctx.whole else torch.zeros_like(zx)
        dy, dnorm = ops.mixer_norm_bwd(y, zx, norm_w, dout, dzx, ctx.eps, offsets)
        du, dbias, dalog, dd = ops.mixer_scan_bwd(u, zx, dt_bias, A_log, D, dy, dzx, offsets)
        dw, db = ops.mixer_conv_bwd(zx, conv_w, conv_b, du, dzx, offsets)
        grads = (dzx, dw, db, dbias, dalog, dd, dnorm)
        return (*(g if need else None for g, need in zip(grads, ctx.needs_input_grad)),
                None, None, None)


class Mamba2Mixer(torch.nn.Module):
    """What stands between in_proj and out_proj of a Mamba-2 block in training:
    the part the paper leaves unquantized (Sec. 3.2).  nheads heads of 64
    channels, 128 states, one group of B and C, four convolution taps.

    forward(zxbcdt, offsets=None): in_proj's output, bfloat16 or float32,
    [L, Z] or [batch, L, Z] (a sequence a row), or with offsets (int32
    [nseq + 1] on the GPU) packed sequences [T, Z] (65535 sequences at most); returns out_proj's input,
    bfloat16 [..., d_inner].  Sequences begin with zero states; rows outside
    the offsets come out zero and have no gradient."""

    PARAMS = ("conv_w", "conv_b", "dt_bias", "A_log", "D", "norm_w")

    def __init__(self, nheads: int, eps: float = 1e-5, device: Optional[torch.device] = None):
        super().__init__()
        if nheads < 1:
            raise ValueError("nheads must be at least 1")
        self.nheads, self.eps = nheads, eps
        self.d_inner = nheads * ops.MIXER_HEADDIM
        cd = self.d_inner + 2 * ops.MIXER_DSTATE
        f32 = dict(dtype=torch.float32, device=device)
        step = torch.exp(torch.empty(nheads, **f32).uniform_(math.log(1e-3), math.log(1e-1)))
        par = dict(conv_w=torch.empty((cd, 4), **f32).uniform_(-0.5, 0.5),
                   conv_b=torch.empty((cd,), **f32).uniform_(-0.5, 0.5),
                   dt_bias=step + torch.log(-torch.expm1(-step)),  # softplus^-1(step)
                   A_log=torch.log(torch.empty(nheads, **f32).uniform_(1.0, 16.0)),
                   D=torch.ones(nheads, **f32), norm_w=torch.ones(self.d_inner, **f32))
        for name in self.PARAMS:
            setattr(self, name, torch.nn.Parameter(par[name]))

    def forward(self, zxbcdt: torch.Tensor,
                offsets: Optional[torch.Tensor] = None) -> torch.Tensor:
        if zxbcdt.dim() not in (2, 3):
            raise ValueError(f"zxbcdt must be [L, Z] or [batch, L, Z], got {tuple(zxbcdt.shape)}")
        lead, whole = zxbcdt.shape[:-1], offsets is None
        if offsets is not None:
            if zxbcdt.dim() != 2:
                raise ValueError("packed sequences (offsets) are [T, Z]")
        elif zxbcdt.dim() == 3 and lead[0] != 1 and lead.numel():
            offsets = torch.arange(0, lead.numel() + 1, lead[1], dtype=torch.int32,
                                   device=zxbcdt.device)
        out = Mamba2MixerFn.apply(zxbcdt.reshape(-1, zxbcdt.shape[-1]),
                                  *(getattr(self, n) for n in self.PARAMS), offsets, self.eps,
                                  whole)
        return out.reshape(*lead, self.d_inner)

    def decode_params(self) -> dict:
        """The arrays ``Mamba2Decoder``'s mixer(l) gives."""
        return {n: getattr(self, n).detach() for n in self.PARAMS}

    def extra_repr(self) -> str:
        return f"nheads={self.nheads}, d_inner={self.d_inner}, eps={self.eps}"


class EmbeddingFn(torch.autograd.Function):
    """Rows of a weight times a scale (``tm_embed``, ``tm_embed_bwd``)."""

    @staticmethod
    def forward(ctx, ids, weight, scale):
        ctx.save_for_backward(ids)
        ctx.vocab, ctx.scale, ctx.dtype = weight.shape[0], scale, weight.dtype
        return ops.embed(ids, weight.detach().contiguous(), scale)

    @staticmethod
    @once_differentiable
    def backward(ctx, de):
        (ids,) = ctx.saved_tensors
        dw = ops.embed_bwd(ids, de.to(torch.float32).contiguous(), ctx.vocab, ctx.scale)
        return None, dw.to(ctx.dtype), None


class Embedding(torch.nn.Module):
    """Token embedding whose output is the float32 residual stream, scaled:
    forward(ids int32 or int64 [...]) -> float32 [..., width].  Ids outside the
    vocabulary are padding: rows of zeros without a gradient.  The gradient of
    the weight adds the tokens of a row in ascending order, so that repeated
    steps give the same bits."""

    def __init__(self, vocab: int, width: int, scale: float = 1.0,
                 device: Optional[torch.device] = None, dtype: torch.dtype = torch.float32):
        super().__init__()
        self.scale = scale
        self.weight = torch.nn.Parameter(torch.empty((vocab, width), device=device, dtype=dtype))
        torch.nn.init.normal_(self.weight, 0.0, 0.02)

    def forward(self, ids: torch.Tensor) -> torch.Tensor:
        e = EmbeddingFn.apply(ids.reshape(-1).contiguous(), self.weight, self.scale)
        return e.reshape(*ids.shape, self.weight.shape[1])

    def extra_repr(self) -> str:
        return f"{self.weight.shape[0]}, {self.weight.shape[1]}, scale={self.scale}"


def flops_per_step(tokens: int, layer: TernaryLinear) -> float:
    """Algorithmic flops of one forward + straight-through backward (three
    dense products of 2 * tokens * in * out each; zeros not discounted)."""
    return 3.0 * 2.0 * tokens * layer.in_features * layer.out_features


__all__ = ["SCALE_MODES", "TernaryLinear", "TernaryLinearFn", "Mamba2Mixer", "Mamba2MixerFn",
           "Embedding", "EmbeddingFn", "flops_per_step"]
