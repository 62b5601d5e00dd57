"""Performance cases of what stands between a transformer block's MXFP4 linear layers, and of what it keeps for
the backward pass.

A case is a dict of plain values.  Its "kind" names the way a pass goes:

  norm         residual_norm, forward only: h = rho x + sigma g . post(u), y = pre(h)
  norm_serve   the same with y as MXFP4 codes, which go into the next linear layer's product
  norm_train   forward and backward through autograd: h, y and every gradient; with "ckpt" h and u are kept in 8 bits
  act_serve    activation of a product's result with MXFP4 codes out, and the next linear layer's product
  act_train    activation, forward and backward, its input kept in 8 bits
  pack         mx_checkpoint_pack and mx_checkpoint_unpack of one tensor

`x` is the type of the residual stream, `u` that of the branch (and of y), `w` that of norm parameters and gate.
`gates` is the number of gate rows: 0 no gate, 1 one for all, else one for each run of tokens / gates rows.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}
EPS = 1e-6


def listed():
    return [
        # one token of a generated text: the end of one block, the start of the next, and its projection
        dict(name="norm_serve_1_token", kind="norm_serve", tokens=1, d=1024, out=1024, norm="rms", post=True, gates=0, x="bf16"),
        # a batch of prompts through the norms around a wide model's block
        dict(name="norm_prompt_wide", kind="norm", tokens=4096, d=8192, norm="rms", post=True, gates=0, rho=1.0, sigma=0.5,
             x="bf16", u="bf16", w="bf16"),
        # ViT-B on 256 images: residual with a learned gate for each channel, LayerNorm, inputs kept in 8 bits
        dict(name="norm_train_base_b256", kind="norm_train", tokens=256 * 197, d=768, norm="layer", post=False, gates=1, rho=1.0,
             sigma=1.0, x="bf16", u="bf16", w="bf16", ckpt=True),
        # a language model's micro-batch with norms on both sides of each block and a scaled residual
        dict(name="norm_train_sandwich", kind="norm_train", tokens=16384, d=4096, norm="rms", post=True, gates=0, rho=1.25,
             sigma=1.0, x="bf16", u="bf16", w="bf16", ckpt=True),
        # ViT-S on 128 images in FP32, the gate computed for each image, inputs kept as they are
        dict(name="norm_train_small_gate_f32", kind="norm_train", tokens=128 * 197, d=384, norm="layer", post=True, gates=128,
             rho=1.0, sigma=1.0, x="f32", u="f32", w="f32", ckpt=False),
        # a last, partial batch and an odd width: FP32 stream, bf16 branch
        dict(name="norm_train_ragged", kind="norm_train", tokens=50 * 197, d=1001, norm="rms", post=True, gates=1, rho=1.0,
             sigma=0.7, x="f32", u="bf16", w="bf16", ckpt=True),
        # a decoding batch of 16 through the gated MLP's activation and its second projection
        dict(name="act_serve_16_tokens", kind="act_serve", tokens=16, f=4096, out=1024, act="silu", gated=True, x="bf16"),
        # ViT-L's MLP on 256 images
        dict(name="act_train_gelu_large", kind="act_train", tokens=256 * 197, f=4096, act="gelu", gated=False, x="bf16"),
        # a language model's gated MLP
        dict(name="act_train_silu_gated", kind="act_train", tokens=16384, f=8192, act="silu", gated=True, x="bf16"),
        # odd width, FP32, gated GELU
        dict(name="act_train_ragged_f32", kind="act_train", tokens=50 * 197, f=1537, act="gelu", gated=True, x="f32"),
        # an activation kept in 8 bits over a training step: ViT-L's stream, and one image in FP32 at an odd width
        dict(name="pack_large_b256", kind="pack", tokens=256 * 197, d=1024, x="bf16"),
        dict(name="pack_1_image_f32", kind="pack", tokens=197, d=1000, x="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width over the range's logarithm: whole groups of 32, whole vectors of 8, or any."""
    d, r = _log_int(rng, lo, hi), rng.random()
    return max(32, d // 32 * 32) if r < 0.6 else max(8, d // 8 * 8) if r < 0.75 else d


def draw(rng):
    kind = rng.choice(["norm", "norm_serve", "norm_train", "norm_train", "norm_train", "act_serve", "act_train", "act_train", "pack"])
    tokens = _log_int(rng, 1, 50432)
    if kind in ("norm_serve", "act_serve"):
        c = dict(kind=kind, tokens=min(tokens, 4096), out=32 * _log_int(rng, 4, 128), x="bf16")
        width = 32 * _log_int(rng, 4, 256)
        if kind == "norm_serve":
            return dict(c, d=width, norm=rng.choice(["rms", "layer"]), post=rng.random() < 0.6, gates=rng.choice([0, 1]))
        return dict(c, f=width, act=rng.choice(["silu", "gelu"]), gated=rng.random() < 0.7)
    if kind == "act_train":
        f, gated = _width(rng, 128, 16384), rng.random() < 0.5
        return dict(kind=kind, tokens=max(1, min(tokens, (1 << 27) // f)), f=f, act=rng.choice(["silu", "gelu"]), gated=gated,
                    x=rng.choice(["bf16", "bf16", "f32"]))
    d = _width(rng, 64, 16384)
    tokens = max(1, min(tokens, (1 << 25) // d))
    if kind == "pack":
        return dict(kind=kind, tokens=tokens, d=d, x=rng.choice(["bf16", "f32"]))
    x, u = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
    gates = rng.choice([0, 1, 1, 2])
    if gates == 2:                                        # runs of equal length: sequences of a batch
        run = _log_int(rng, 1, tokens)
        gates = max(1, tokens // run)
        tokens = gates * run
    c = dict(kind=kind, tokens=tokens, d=d, norm=rng.choice(["rms", "layer"]), post=rng.random() < 0.6, gates=gates,
             rho=rng.choice([1.0, 1.0, 1.25]), sigma=rng.choice([1.0, 0.5]), x=x, u=u)
    if kind == "norm":
        return dict(c, w=rng.choice(["f32", "bf16"]))
    # parameters of the branch's type; what is kept of an FP32 stream in 8 bits goes with bf16 parameters
    c["ckpt"] = u == "bf16" and rng.random() < 0.7
    c["w"] = u
    return c


# ---- inputs -------------------------------------------------------------------------------------
# Streams are normal with one channel in a hundred twenty times larger, branches normal, weights of a norm near one,
# gates around a half, linear weights normal with deviation 0.02 (as MXFP4 codes and as the values these stand for), output
# gradients Student-t with three degrees of freedom times 1e-3.

def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _stream(g, n, d):
    x = _randn(g, n, d)
    x[:, torch.randperm(d, generator=g, device="cuda")[: max(1, d // 100)]] *= 20.0
    return x


def _grads(g, n, c):
    chi = _randn(g, n, c).square_()
    for _ in range(2):
        chi += _randn(g, n, c).square_()
    return _randn(g, n, c).div_((chi / 3.0).sqrt_()).mul_(1e-3)


def _packed_weight(g, rows, cols):
    """A linear layer's weight as a serving program holds it: codes, scale bytes, and the values they stand for."""
    index, s = _fp4(_randn(g, rows, cols) * 0.02)
    magnitude = (index - 7).abs()
    code = (magnitude + 8 * (index < 7)).to(torch.uint8)
    codes = (code[:, 0::2] | (code[:, 1::2] << 4)).contiguous()
    return codes, (s + 127).to(torch.uint8), _fp4_value(index, s)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind, n, st = case["kind"], case["tokens"], {"case": case}
    if kind == "pack":
        st["x"] = _stream(g, n, case["d"]).to(_TYPES[case["x"]])
        return st
    if kind in ("act_serve", "act_train"):
        width = case["f"] * (2 if case["gated"] else 1)
        st["p"] = (_randn(g, n, width) * 1.5).to(_TYPES[case["x"]])
        if kind == "act_serve":
            st["wq"], st["ws"], st["w"] = _packed_weight(g, case["out"], case["f"])
        else:
            st["p"].requires_grad_(True)
            st["da"] = _grads(g, n, case["f"]).to(_TYPES[case["x"]])
        return st
    d, xt = case["d"], _TYPES[case["x"]]
    ut, wt = _TYPES[case.get("u", case["x"])], _TYPES[case.get("w", case["x"])]
    st["x"], st["u"] = _stream(g, n, d).to(xt), (_randn(g, n, d) * 0.7).to(ut)
    names = ["pre_weight"] + (["post_weight"] if case["post"] else [])
    if case["norm"] == "layer":
        names += ["pre_bias"] + (["post_bias"] if case["post"] else [])
    st["params"] = {k: ((k.endswith("weight")) + 0.1 * _randn(g, d)).to(wt) for k in names}
    if case["gates"]:
        shape = (d,) if case["gates"] == 1 else (case["gates"], d)
        st["params"]["gate"] = (0.5 + 0.25 * _randn(g, *shape)).to(wt)
    if kind == "norm_serve":
        st["wq"], st["ws"], st["w"] = _packed_weight(g, case["out"], d)
    if kind == "norm_train":
        for t in (st["x"], st["u"], *st["params"].values()):
            t.requires_grad_(True)
        st["dh"], st["dy"] = _grads(g, n, d).to(xt), _grads(g, n, d).to(ut)
    return st


# ---- the operators in their plain form ------------------------------------------------------------

def _fp4(x):
    """(index into the 15 values, exponent) of MXFP4: groups of 32 along the columns, the smallest 2^s that leaves no
    magnitude above 6, nearest value, ties to the larger one."""
    groups = x.view(x.shape[0], -1, 32)
    m, e = torch.frexp(groups.abs().amax(-1))
    s = torch.where(m == 0, -29, e - 3 + (m > 0.75).int())
    edges = torch.tensor([-5, -3.5, -2.5, -1.75, -1.25, -0.75, -0.25, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5], device=x.device, dtype=x.dtype)
    index = torch.bucketize(torch.ldexp(groups, -s.unsqueeze(-1)), edges, right=True)
    return index.view(x.shape), s


def _fp4_value(index, s):
    values = torch.tensor([-6, -4, -3, -2, -1.5, -1, -0.5, 0, 0.5, 1, 1.5, 2, 3, 4, 6], device=index.device, dtype=torch.float32)
    return torch.ldexp(values[index].view(index.shape[0], -1, 32), s.unsqueeze(-1)).view(index.shape)


def _eight_bits(x):
    """x (FP32) as its 8-bit checkpoint holds it: groups of 32 along the columns (the last one may be shorter), the
    smallest 2^s that leaves no magnitude above 448, E4M3 elements, nearest even."""
    n, d = x.shape
    groups = torch.nn.functional.pad(x, (0, -d % 32)).view(n, -1, 32)
    m, e = torch.frexp(groups.abs().amax(-1, keepdim=True))
    s = e - 9 + (m > 0.875).int()
    q = torch.ldexp(groups, -s).to(torch.float8_e4m3fn).float()
    return torch.ldexp(q, s).view(n, -1)[:, :d]


def _statistics(a, norm):
    mean = a.mean(-1, keepdim=True) if norm == "layer" else torch.zeros_like(a[:, :1])
    return mean, 1.0 / ((a - mean).square().mean(-1, keepdim=True) + EPS).sqrt()


def _gate_rows(case, gate):
    """The gate's row of every token, or one row for all."""
    return gate.view(-1, case["d"]).repeat_interleave(case["tokens"] // case["gates"], 0) if case["gates"] > 1 else gate.view(1, -1)


def _plain_norm(case, x, u, params):
    p = {k: v.detach().float() for k, v in params.items()}
    x, u = x.detach().float(), u.detach().float()
    v, stats_u = u, None
    if case["post"]:
        stats_u = _statistics(u, case["norm"])
        v = (u - stats_u[0]) * stats_u[1] * p["post_weight"] + p.get("post_bias", 0.0)
    branch = v * _gate_rows(case, p["gate"]) if case["gates"] else v
    # the next norm works on the stream as it is stored
    h = (case.get("rho", 1.0) * x + case.get("sigma", 1.0) * branch).to(_TYPES[case["x"]]).float()
    stats_h = _statistics(h, case["norm"])
    y = (h - stats_h[0]) * stats_h[1] * p["pre_weight"] + p.get("pre_bias", 0.0)
    return h, y, stats_h, stats_u


def _plain_norm_backward(case, st, h, stats_h, stats_u):
    """Gradients from what was kept: h and u as stored, and the statistics of the forward pass."""
    p = {k: v.detach().float() for k, v in st["params"].items()}
    u, dy, dh = st["u"].detach().float(), st["dy"].float(), st["dh"].float()
    if case["ckpt"]:
        h, u = _eight_bits(h), _eight_bits(u)
    layer, grads = case["norm"] == "layer", {}

    def normalised(a, stats, weight, da):
        """(gradient of the norm's input, normalised input) for the output's gradient da."""
        a_hat, b = (a - stats[0]) * stats[1], da * weight
        mean = b.mean(-1, keepdim=True) if layer else 0.0
        return stats[1] * (b - mean - a_hat * (b * a_hat).mean(-1, keepdim=True)), a_hat

    through, h_hat = normalised(h, stats_h, p["pre_weight"], dy)
    grads["pre_weight"] = (dy * h_hat).sum(0)
    if layer:
        grads["pre_bias"] = dy.sum(0)
    dh = dh + through
    dx, dbranch = case["rho"] * dh, case["sigma"] * dh
    dv = dbranch
    if case["gates"]:
        dv = dbranch * _gate_rows(case, p["gate"])
    v = u
    if case["post"]:
        du, u_hat = normalised(u, stats_u, p["post_weight"], dv)
        grads["post_weight"] = (dv * u_hat).sum(0)
        if layer:
            grads["post_bias"] = dv.sum(0)
        v = u_hat * p["post_weight"] + p.get("post_bias", 0.0)
    else:
        du = dv
    if case["gates"]:
        grads["gate"] = (dbranch * v).view(case["gates"], -1, case["d"]).sum(1).view_as(p["gate"])
    return dx.to(st["x"].dtype), du.to(st["u"].dtype), {k: grads[k].to(t.dtype) for k, t in st["params"].items()}


def _act(kind, x):
    """(activation, its derivative)."""
    if kind == "silu":
        s = 1.0 / (1.0 + torch.exp(-x))
        return x * s, s * (1.0 + x * (1.0 - s))
    phi = 0.5 * torch.erfc(x * -math.sqrt(0.5))
    return x * phi, phi + x * torch.exp(-0.5 * x * x) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain_act(case, p):
    if not case["gated"]:
        return _act(case["act"], p)[0]
    return _act(case["act"], p[:, : case["f"]])[0] * p[:, case["f"]:]


def _plain_act_backward(case, p, da):
    if not case["gated"]:
        return da * _act(case["act"], _eight_bits(p))[1]
    gate, up = _eight_bits(p[:, : case["f"]].contiguous()), _eight_bits(p[:, case["f"]:].contiguous())
    a, slope = _act(case["act"], gate)
    return torch.cat([da * up * slope, da * a], 1)


# ---- one pass -----------------------------------------------------------------------------------

def run(st):
    return _RUN[st["case"]["kind"]](st["case"], st)


def _norm_options(case):
    return dict(norm=case["norm"], post=case["post"], residual_scale=case.get("rho", 1.0), branch_scale=case.get("sigma", 1.0), eps=EPS)


def _run_norm(case, st):
    if own:
        import paper_2502_20853_amd as mx
        return mx.residual_norm(st["x"], st["u"], **st["params"], **_norm_options(case))
    h, y, _, _ = _plain_norm(case, st["x"], st["u"], st["params"])
    return h.to(st["x"].dtype), y.to(st["u"].dtype)


def _run_norm_serve(case, st):
    if own:
        import paper_2502_20853_amd as mx
        h, (codes, scales) = mx.residual_norm(st["x"], st["u"], **st["params"], packed=True, **_norm_options(case))
        return h, mx.mx_linear_fwd(codes, scales, st["wq"], st["ws"], out_dtype=torch.bfloat16)
    h, y, _, _ = _plain_norm(case, st["x"], st["u"], st["params"])
    return h.to(st["x"].dtype), (_fp4_value(*_fp4(y)) @ st["w"].t()).to(torch.bfloat16)


def _run_norm_train(case, st):
    if own:
        import paper_2502_20853_amd as mx
        h, y = mx.residual_norm(st["x"], st["u"], **st["params"], checkpoint=case["ckpt"], **_norm_options(case))
        grads = torch.autograd.grad((h, y), (st["x"], st["u"], *st["params"].values()), (st["dh"], st["dy"]))
        return h.detach(), y.detach(), grads[0], grads[1], dict(zip(st["params"], grads[2:]))
    h, y, stats_h, stats_u = _plain_norm(case, st["x"], st["u"], st["params"])
    dx, du, grads = _plain_norm_backward(case, st, h, stats_h, stats_u)
    return h.to(st["x"].dtype), y.to(st["u"].dtype), dx, du, grads


def _run_act_serve(case, st):
    if own:
        import paper_2502_20853_amd as mx
        codes, scales = mx.activation(st["p"], case["act"], gated=case["gated"], packed=True)
        return mx.mx_linear_fwd(codes, scales, st["wq"], st["ws"], out_dtype=torch.bfloat16)
    return (_fp4_value(*_fp4(_plain_act(case, st["p"].float()))) @ st["w"].t()).to(torch.bfloat16)


def _run_act_train(case, st):
    if own:
        import paper_2502_20853_amd as mx
        a = mx.activation(st["p"], case["act"], gated=case["gated"], checkpoint=True)
        return a.detach(), torch.autograd.grad(a, st["p"], st["da"])[0]
    p = st["p"].detach().float()
    return _plain_act(case, p).to(st["p"].dtype), _plain_act_backward(case, p, st["da"].float()).to(st["p"].dtype)


def _run_pack(case, st):
    if own:
        import paper_2502_20853_amd as mx
        codes, scales = mx.mx_checkpoint_pack(st["x"])
        return mx.mx_checkpoint_unpack(codes, scales, case["d"], st["x"].dtype)
    return _eight_bits(st["x"].float()).to(st["x"].dtype)


_RUN = {"norm": _run_norm, "norm_serve": _run_norm_serve, "norm_train": _run_norm_train, "act_serve": _run_act_serve,
        "act_train": _run_act_train, "pack": _run_pack}


# ---- the definitions in 64 bits, apart from the above ----------------------------------------------

def _grid64(x, top, mantissa, lowest):
    """x (float64) rounded to a format of `mantissa` bits behind the point, magnitudes up to `top`, exponents from
    `lowest` on, under one power of two for each 32 columns; nearest, ties to even."""
    n, d = x.shape
    full = torch.zeros((n, (d + 31) // 32 * 32), dtype=torch.float64, device=x.device)
    full[:, :d] = x
    full = full.view(n, -1, 32)
    peak = full.abs().max(-1, keepdim=True).values
    s = torch.ceil(torch.log2(peak.clamp_min(2.0 ** -140) / top))
    s = torch.where(peak > top * torch.exp2(s), s + 1, torch.where(peak <= top * torch.exp2(s - 1), s - 1, s))
    t = full / torch.exp2(s)
    e = torch.floor(torch.log2(t.abs().clamp_min(2.0 ** -40))).clamp_min(lowest)
    step = torch.exp2(e - mantissa)
    return t, s, step


def _eight64(x):
    t, s, step = _grid64(x, 448.0, 3, -6)
    return (torch.round(t / step) * step * torch.exp2(s)).view(x.shape[0], -1)[:, : x.shape[1]]


def _four64(x):
    t, s, step = _grid64(x, 6.0, 1, 0)
    return (torch.floor(t / step + 0.5) * step * torch.exp2(s)).view(x.shape)        # ties to the larger value


def _norm64(a, norm, weight, bias):
    centred = a - a.mean(1, keepdim=True) if norm == "layer" else a
    r = (centred.pow(2).mean(1, keepdim=True) + EPS).rsqrt()
    return centred * r * weight + (0 if bias is None else bias), r, a.mean(1, keepdim=True) if norm == "layer" else 0.0


def _slope64(kind, x):
    if kind == "silu":
        s = torch.sigmoid(x)
        return s + x * s * torch.sigmoid(-x)
    return torch.special.ndtr(x) + x * torch.exp(-x * x / 2) / (2 * math.pi) ** 0.5


def _value64(kind, x):
    return x * (torch.sigmoid(x) if kind == "silu" else torch.special.ndtr(x))


def _backward64(da, a, r, mean, weight, layer):
    """(gradient of a norm's input, normalised input): the product with the norm's Jacobian, at the statistics given."""
    a_hat, c = (a - mean) * r, da * weight
    d = a.shape[1]
    inner = (c * a_hat).sum(1, keepdim=True) / d
    return (c - (c.sum(1, keepdim=True) / d if layer else 0) - a_hat * inner) * r, a_hat


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    f64 = lambda t: t.detach().double()  # noqa: E731
    if kind == "pack":
        return _eight64(f64(st["x"]))
    if kind in ("act_serve", "act_train"):
        p, f = f64(st["p"]), case["f"]
        a = _value64(case["act"], p[:, :f]) * (p[:, f:] if case["gated"] else 1.0)
        if kind == "act_serve":
            return _four64(a) @ f64(st["w"]).t()
        da = f64(st["da"])
        if not case["gated"]:
            return a, da * _slope64(case["act"], _eight64(p))
        gate, up = _eight64(p[:, :f]), _eight64(p[:, f:])
        return a, torch.cat([da * up * _slope64(case["act"], gate), da * _value64(case["act"], gate)], 1)
    q = {k: f64(v) for k, v in st["params"].items()}
    x, u, layer = f64(st["x"]), f64(st["u"]), case["norm"] == "layer"
    rho, sigma = case.get("rho", 1.0), case.get("sigma", 1.0)
    v, r_u, mean_u = _norm64(u, case["norm"], q["post_weight"], q.get("post_bias")) if case["post"] else (u, None, None)
    per = case["tokens"] // max(1, case["gates"])
    g = q["gate"].reshape(-1, case["d"])[torch.arange(case["tokens"], device=x.device) // per] if case["gates"] else torch.ones_like(x[:1])
    h = rho * x + sigma * g * v
    kept = h.to(st["x"].dtype).double()
    y, r_h, mean_h = _norm64(kept, case["norm"], q["pre_weight"], q.get("pre_bias"))
    if kind == "norm_serve":
        return h, _four64(y) @ f64(st["w"]).t()
    if kind == "norm":
        return h, y
    u_kept = u
    if case["ckpt"]:
        kept, u_kept = _eight64(kept), _eight64(u)
    dy, grads = f64(st["dy"]), {}
    back, h_hat = _backward64(dy, kept, r_h, mean_h, q["pre_weight"], layer)
    dh = f64(st["dh"]) + back
    dv = sigma * g * dh
    grads["pre_weight"], grads["pre_bias"] = (dy * h_hat).sum(0), dy.sum(0)
    du, v = dv, u_kept
    if case["post"]:
        du, u_hat = _backward64(dv, u_kept, r_u, mean_u, q["post_weight"], layer)
        grads["post_weight"], grads["post_bias"] = (dv * u_hat).sum(0), dv.sum(0)
        v = u_hat * q["post_weight"] + q.get("post_bias", 0.0)
    if case["gates"]:
        grads["gate"] = torch.stack([part.sum(0) for part in (sigma * dh * v).split(per)]).view_as(q["gate"])
    return h, y, rho * dh, du, {k: grads[k] for k in q}


# ---- what a pass cannot do without --------------------------------------------------------------

def work(case):
    kind, n = case["kind"], case["tokens"]
    eight = 1 + 1 / 32
    xb, ub = _BYTES[case["x"]], _BYTES[case.get("u", case["x"])]
    if kind == "pack":
        # packed, and read back
        return {"bytes": n * case["d"] * (2 * xb + 2 * eight), "flops": 4.0 * n * case["d"]}
    if kind in ("act_serve", "act_train"):
        a = n * case["f"]
        p = a * (2 if case["gated"] else 1)
        if kind == "act_serve":
            return {"bytes": p * xb + case["out"] * case["f"] * 17 / 32 + n * case["out"] * 2, "flops": 2.0 * n * case["f"] * case["out"] + 12.0 * a}
        # forward: P in, A and the 8-bit P out; backward: dA and the 8-bit P in, dP out
        return {"bytes": p * xb + a * xb + 2 * p * eight + a * xb + p * xb, "flops": 50.0 * a}
    e, params = n * case["d"], _BYTES[case.get("w", case["x"])] * case["d"] * (2 + max(1, case["gates"]))
    if kind == "norm_serve":
        return {"bytes": e * (2 * xb + ub) + params + case["out"] * case["d"] * 17 / 32 + n * case["out"] * 2,
                "flops": 2.0 * e * case["out"] + 16.0 * e}
    forward = e * (2 * xb + 2 * ub) + params
    if kind == "norm":
        return {"bytes": forward, "flops": 16.0 * e}
    # backward: both gradients and what was kept of h and, with a norm or a gate on the branch, of u; dx and du out
    of_u = case["post"] or case["gates"] > 0
    kept = e * eight * (2 + 2 * of_u) if case["ckpt"] else e * (xb + ub * of_u)
    return {"bytes": forward + e * (2 * xb + 2 * ub) + kept + 2 * params, "flops": 50.0 * e}
