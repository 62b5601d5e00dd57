"""Definitions in 64 bits of the operators between the linear layers, with bounds on what FP32 arithmetic may add.

Every function works on float64 CPU tensors.  A bound counts roundings: EPS is half a step of FP32 at 1, each of the
kernels' operations adds at most one, and a sum of n terms at most n of them times the sum of the magnitudes.
"""
import torch

EPS = 2.0 ** -24
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}          # torch.finfo(t).eps / 2


def eight_bits(x):
    """The values that the 8-bit checkpoint of x stands for: decided by comparisons with the E4M3 values themselves."""
    x = x.double()
    n, d = x.shape
    pad = torch.zeros((n, -d % 32), dtype=torch.float64)
    g = torch.cat([x, pad], 1).view(n, -1, 32)
    top = g.abs().amax(-1, keepdim=True)
    s = torch.full_like(top, -127.0)
    for e in range(-127, 121):                                              # the smallest power of two that fits
        s = torch.where(top > 448.0 * 2.0 ** e, float(e + 1), s)
    t = (g / torch.exp2(s)).abs()
    values = torch.tensor([m / 8 * 2.0 ** -6 for m in range(8)] + [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8)][:-1],
                          dtype=torch.float64)                              # the pattern 127 is no number
    hi = torch.searchsorted(values, t.contiguous()).clamp(max=len(values) - 1)
    lo = (hi - 1).clamp(min=0)
    a, b = t - values[lo], values[hi] - t
    pick = torch.where((b < a) | ((b == a) & (hi % 2 == 0)), hi, lo)
    q = torch.where(t == values[hi], values[hi], values[pick])
    return (torch.sign(g) * q * torch.exp2(s)).view(n, -1)[:, :d], (s.squeeze(-1) + 127).to(torch.uint8)


def stats(a, layer, eps):
    mean = a.mean(1, keepdim=True) if layer else torch.zeros_like(a[:, :1])
    return mean, ((a - mean).square().mean(1, keepdim=True) + eps) ** -0.5


def per_row(gate, rows):
    """The gate's row of every row (None: ones)."""
    g = gate.reshape(-1, gate.shape[-1])
    return g.repeat_interleave(rows // g.shape[0], 0)


def norm(a, layer, eps, w, b):
    """(value, scale of its roundings)."""
    mean, r = stats(a, layer, eps)
    w = torch.ones_like(a[:1]) if w is None else w
    b = torch.zeros_like(a[:1]) if b is None else b
    value = (a - mean) * r * w + b
    # the reciprocal deviation carries half of its sum's roundings, the mean those of its own
    return value, ((a - mean).abs() + (a.abs().mean(1, keepdim=True) if layer else 0)) * r * w.abs() + b.abs()


def forward_h(x, u, p, o):
    """(h before it is stored, scale of its roundings).  p: parameters by name, o: options by name."""
    v, scale = (norm(u, o["layer"], o["eps"], p.get("post_weight"), p.get("post_bias")) if o["post"] else (u, u.abs()))
    g = per_row(p["gate"], x.shape[0]) if "gate" in p else torch.ones_like(x[:1])
    return o["rho"] * x + o["sigma"] * g * v, (o["rho"] * x).abs() + (o["sigma"] * g).abs() * scale


def backward(x_shape, h, u, h_kept, u_kept, dh, dy, p, o):
    """Gradients by name as (value, scale of the roundings, number of rows summed).  h, u give the statistics; h_kept, u_kept
    are the values that the backward pass sees."""
    n, d = x_shape
    out = {}
    one = torch.ones((1, d), dtype=torch.float64)
    t, t_scale = dh, dh.abs()
    if dy is not None:
        mean, r = stats(h, o["layer"], o["eps"])
        w = p.get("pre_weight", one)
        hn, b = (h_kept - mean) * r, dy * w
        hs = (h_kept.abs() + mean.abs()) * r
        m0 = b.mean(1, keepdim=True) if o["layer"] else 0.0
        t = t + r * (b - m0 - hn * (b * hn).mean(1, keepdim=True))
        t_scale = t_scale + r * (b.abs() + (b.abs().mean(1, keepdim=True) if o["layer"] else 0) + hs * (b.abs() * hs).mean(1, keepdim=True))
        out["pre_weight"] = ((dy * hn).sum(0), (dy.abs() * hs).sum(0), n)
        out["pre_bias"] = (dy.sum(0), dy.abs().sum(0), n)
    out["x"] = (o["rho"] * t, abs(o["rho"]) * t_scale, 1)
    if u is None:
        return out
    g = per_row(p["gate"], n) if "gate" in p else one
    e, e_scale = o["sigma"] * t, abs(o["sigma"]) * t_scale
    dv, dv_scale = e * g, e_scale * g.abs()
    v, v_scale = u_kept, u_kept.abs()
    if o["post"]:
        mean, r = stats(u, o["layer"], o["eps"])
        w = p.get("post_weight", one)
        un, us = (u_kept - mean) * r, (u_kept.abs() + mean.abs()) * r
        bias = p.get("post_bias", torch.zeros_like(one))
        v, v_scale = un * w + bias, us * w.abs() + bias.abs()
        c, c_scale = dv * w, dv_scale * w.abs()
        m0 = c.mean(1, keepdim=True) if o["layer"] else 0.0
        du = r * (c - m0 - un * (c * un).mean(1, keepdim=True))
        du_scale = r * (c_scale + (c_scale.mean(1, keepdim=True) if o["layer"] else 0) + us * (c_scale * us).mean(1, keepdim=True))
        out["post_weight"] = ((dv * un).sum(0), (dv_scale * us).sum(0), n)
        out["post_bias"] = (dv.sum(0), dv_scale.sum(0), n)
    else:
        du, du_scale = dv, dv_scale
    out["u"] = (du, du_scale, 1)
    if "gate" in p:
        gates = p["gate"].reshape(-1, d).shape[0]
        sums = lambda a: a.view(gates, n // gates, d).sum(1)
        out["gate"] = (sums(e * v), sums(e_scale * v_scale), n // gates)
    return out


def act(kind, x):
    """(act(x), act'(x))."""
    if kind == "silu":
        s = torch.sigmoid(x)
        return x * s, s * (1 + x * torch.sigmoid(-x))
    phi = torch.special.erfc(x * -0.5 ** 0.5) / 2                           # not 1 + erf, which cancels in the tail
    return x * phi, phi + x * torch.exp(-x * x / 2) * (2 * torch.pi) ** -0.5


def four_bits(values, scale_mode_floor=False):
    """MXFP4 codes and scale bytes of rows, nearest value, ties to the larger one, by comparison with the 15 values."""
    n, d = values.shape
    g = values.double().view(n, -1, 32)
    top = g.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(torch.where(top == 0, 1e-8, top))
    s = (e - 3 + (0 if scale_mode_floor else (m > 0.75).int())).clamp(min=-127)
    t = (g / torch.exp2(s.double())).clamp(-6, 6)
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
    mids = (grid[1:] + grid[:-1]) / 2
    up = torch.searchsorted(mids, t.abs().contiguous(), right=True)         # ties away from zero
    down = torch.searchsorted(mids, t.abs().contiguous(), right=False)      # ties toward zero
    neg = torch.signbit(g)
    code = torch.where(neg, down + 8, up)
    return code.view(n, d), (s.squeeze(-1) + 127).to(torch.uint8)
