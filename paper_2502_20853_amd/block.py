"""What stands between the MXFP4 linear layers of a transformer block: the residual around a block with the norms on
both of its sides, and the activation of an MLP.  Each is one kernel in each direction, and each can keep what its
backward pass needs in 8 bits (mx_checkpoint_pack's format) in place of the 16 or 32 that autograd would hold, beside
the 4 bits that MxLinear keeps.  Plumbing only: csrc/mx_torch.cpp makes the calls and carries the autograd graph.
"""
import torch

from . import binding as B

_NORMS = ("rms", "layer")
_ACTS = ("gelu", "silu")


def residual_norm(x, u=None, *, pre_weight=None, pre_bias=None, post_weight=None, post_bias=None, gate=None, norm="rms",
                  pre=True, post=False, residual_scale=1.0, branch_scale=1.0, eps=1e-6, checkpoint=False, packed=False,
                  scale_mode=B.SCALE_TRUNCFREE):
    """(h, y):  h = residual_scale * x + branch_scale * gate * post_norm(u),  y = pre_norm(h).

    x [..., D] is the residual stream and u the block's output; x and h are float32 or bfloat16, u and y bfloat16 or, with
    a float32 stream, float32; D <= 16384.  norm="rms" or "layer" names both norms; post=True norms u first, pre=False
    leaves y out (None).  Without u the call is the norm of x alone and h is x.  y is the norm of h as stored.
    Weights and biases: vectors of D values of one type, None for ones and zeros.
    gate: [D], or one row for each run of rows: leading sizes those of x up to some dimension and ones behind it
    ([B, 1, D] for x [B, T, D]), or [G, D] for a matrix x whose rows G divides.
    checkpoint=True keeps h and u for the backward pass in 8 bits; the gradients are then those at the kept values.
    packed=True (without gradients) returns y as (codes, scales), the round-to-nearest MXFP4 rows that mx_linear_fwd takes.
    """
    if norm not in _NORMS:
        raise ValueError("norm must be 'rms' or 'layer'")
    r = B.host().residual_norm(x, u, pre_weight, pre_bias, post_weight, post_bias, gate, norm == "layer", pre, post,
                               residual_scale, branch_scale, eps, checkpoint, packed, scale_mode)
    return (r[0], (r[1], r[2])) if packed else (r[0], r[1])


def activation(p, kind="gelu", *, gated=False, checkpoint=False, packed=False, scale_mode=B.SCALE_TRUNCFREE):
    """act(p), or gated act(p1) * p2 for p = [p1 | p2] along the last dimension; kind "gelu" (exact) or "silu".

    p [..., F] (gated [..., 2 F]) is float32 or bfloat16.  checkpoint=True keeps p for the backward pass in 8 bits; the
    gradient is then that at the kept values.  packed=True (without gradients) returns (codes, scales), the
    round-to-nearest MXFP4 rows that mx_linear_fwd takes.
    """
    if kind not in _ACTS:
        raise ValueError("kind must be 'gelu' or 'silu'")
    r = B.host().activation(p, kind == "silu", gated, checkpoint, packed, scale_mode)
    return (r[0], r[1]) if packed else r[0]


class MxResidualNorm(torch.nn.Module):
    """residual_norm with its parameters.  gate: None, or the starting value of a learned gate for each channel; a gate
    computed elsewhere goes to forward().  affine=False leaves the norms without weights and biases."""

    def __init__(self, features, norm="rms", pre=True, post=False, gate=None, affine=True, residual_scale=1.0, branch_scale=1.0,
                 eps=1e-6, checkpoint=True, device="cuda", dtype=torch.float32):
        super().__init__()
        if norm not in _NORMS:
            raise ValueError("norm must be 'rms' or 'layer'")
        self.features, self.norm, self.pre, self.post, self.eps = features, norm, pre, post, eps
        self.residual_scale, self.branch_scale, self.checkpoint = residual_scale, branch_scale, checkpoint
        vector = lambda wanted, value: (torch.nn.Parameter(torch.full((features,), float(value), device=device, dtype=dtype))
                                        if wanted else None)
        self.pre_weight, self.post_weight = vector(affine and pre, 1), vector(affine and post, 1)
        self.pre_bias = vector(affine and pre and norm == "layer", 0)
        self.post_bias = vector(affine and post and norm == "layer", 0)
        self.gate = vector(gate is not None, 0 if gate is None else gate)

    def forward(self, x, u=None, gate=None, packed=False):
        """(h, y); without u the pre-norm of x alone (the first block's input), which a module with pre=False has not."""
        if gate is not None and self.gate is not None:
            raise ValueError("this module has a gate of its own")
        if u is None and (gate is not None or not self.pre):
            raise ValueError("without a branch u there is only the pre-norm of x: no gate, and a module with pre=True")
        pre = dict(pre_weight=self.pre_weight, pre_bias=self.pre_bias, norm=self.norm, eps=self.eps, checkpoint=self.checkpoint, packed=packed)
        if u is None:
            return residual_norm(x, **pre)
        return residual_norm(x, u, post_weight=self.post_weight, post_bias=self.post_bias, gate=self.gate if gate is None else gate,
                             pre=self.pre, post=self.post, residual_scale=self.residual_scale, branch_scale=self.branch_scale, **pre)


class MxActivation(torch.nn.Module):
    """activation as a module; checkpoint=True (its input kept in 8 bits) by default."""

    def __init__(self, kind="gelu", gated=False, checkpoint=True):
        super().__init__()
        if kind not in _ACTS:
            raise ValueError("kind must be 'gelu' or 'silu'")
        self.kind, self.gated, self.checkpoint = kind, gated, checkpoint

    def forward(self, p, packed=False):
        return activation(p, self.kind, gated=self.gated, checkpoint=self.checkpoint, packed=packed)
