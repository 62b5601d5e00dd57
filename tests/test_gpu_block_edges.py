"""Operators between the linear layers on the GPU: values that are not finite, arguments that a norm does not read, results
that are zero.  Against the definitions in 64 bits (block_ref), with the bounds of test_gpu_block."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
import block_ref as ref  # noqa: E402
from test_gpu_block import BACKWARD_OPS, BF, F32, check, f64, make, mx  # noqa: E402,F401

pytestmark = pytest.mark.gpu

KINDS = [(BF, BF, BF), (F32, BF, F32), (F32, F32, F32)]


# narrow rows, rows that end inside a vector, two vectors a lane, rows of four, whose backward pass goes in halves
@pytest.mark.parametrize("d", [5, 41, 48, 1001, 1024, 8200, 8203])
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("pre", [False, True])
def test_rows_that_are_not_finite_without_a_gradient_of_y(mx, d, layer, pre):
    """Without a norm behind h, or a gradient of it, the gradient of h is what came in, whatever h holds: a NaN, an infinity,
    squares beyond FP32."""
    n, i = 12, 0
    for post in (False, True):
        for gates in (0, 1, 3):
            for ckpt in (False, True):
                xt, ut, pt = KINDS[i % 3]
                i += 1
                print("no dy", d, layer, pre, post, gates, ckpt, flush=True)
                g = torch.Generator(device="cuda").manual_seed(60 + i)
                x, u, p = make(g, n, d, xt, ut, pt, layer, post, gates)
                x[4, d // 2], x[6, 0], x[9, d - 1], x[10, 0] = float("nan"), float("inf"), 1e30, float("-inf")
                if pre:
                    p["pre_weight"][d // 3] = float("inf")
                else:
                    p = {k: v for k, v in p.items() if not k.startswith("pre")}
                dh = (torch.randn((n, d), generator=g, device="cuda") * 1e-2).to(xt)
                dh[4] = 0
                leaves = {"x": x, "u": u, **p}
                for t in leaves.values():
                    t.requires_grad_(True)
                o = dict(layer=layer, post=post, rho=1.25, sigma=0.7, eps=1e-6)
                h, _ = mx.residual_norm(x, u, **p, norm="layer" if layer else "rms", pre=pre, post=post, residual_scale=1.25, branch_scale=0.7, checkpoint=ckpt)
                grads = torch.autograd.grad(h, list(leaves.values()), dh, allow_unused=True)
                u_kept = ref.eight_bits(f64(u))[0] if ckpt else f64(u)
                p64 = {k: f64(v) for k, v in p.items() if not k.startswith("pre")}
                want = ref.backward((n, d), None, f64(u), None, u_kept, f64(dh), None, p64, o)
                for (name, leaf), got in zip(leaves.items(), grads):
                    if name not in want:
                        assert got is None, name
                        continue
                    value, scale, rows = want[name]
                    check(got, value.view(leaf.shape), scale.view(leaf.shape), BACKWARD_OPS + rows, "d " + name)


@pytest.mark.parametrize("d", [5, 40, 41, 1001, 1024, 8200, 8203])
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("ckpt", [False, True])
def test_infinite_branch_without_a_post_norm(mx, d, layer, ckpt):
    """Without a post-norm u is in the gate's gradient alone: du is what it is elsewhere, and so is the rest of the gate's."""
    n = 12
    for i, gates in enumerate((1, 3, 12)):
        xt, ut, pt = KINDS[i]
        g = torch.Generator(device="cuda").manual_seed(80 + i)
        x, u, p = make(g, n, d, xt, ut, pt, layer, False, gates)
        p = {"gate": p["gate"]}
        u[5, d // 2], u[6, 0] = float("inf"), float("-inf")
        dh = (torch.randn((n, d), generator=g, device="cuda") * 1e-2).to(xt)
        leaves = [t.requires_grad_(True) for t in (x, u, p["gate"])]
        o = dict(layer=layer, post=False, rho=1.25, sigma=0.7, eps=1e-6)
        h, _ = mx.residual_norm(x, u, **p, norm="layer" if layer else "rms", pre=False, residual_scale=1.25, branch_scale=0.7, checkpoint=ckpt)
        dx, du, dgate = torch.autograd.grad(h, leaves, dh)
        # the definition with finite values there: what is a multiple of them is looked at elsewhere only
        infinite = torch.isinf(f64(u))
        u64 = f64(u).masked_fill(infinite, 0.0)
        kept = ref.eight_bits(u64)[0] if ckpt else u64
        want = ref.backward((n, d), None, u64, None, kept, f64(dh), None, {"gate": f64(p["gate"])}, o)
        check(dx, *want["x"][:2], BACKWARD_OPS, "dx")
        check(du, *want["u"][:2], BACKWARD_OPS, "du")
        touched = infinite
        if ckpt:                                          # a group that holds an infinity comes back as NaN as a whole
            touched = torch.nn.functional.pad(infinite, (0, -d % 32)).view(n, -1, 32).any(-1).repeat_interleave(32, 1)[:, :d]
        touched = touched.view(gates, n // gates, d).any(1)
        assert not torch.isfinite(dgate.cpu().view(gates, d)[touched]).any()
        value, scale, rows = want["gate"]
        clean = lambda t: t.cpu().view(gates, d).masked_fill(touched, 0.0)
        check(clean(dgate), clean(value), clean(scale), BACKWARD_OPS + rows, "d gate")


class Call:
    """A forward and a backward pass through the C interface."""

    def __init__(self, mx, n, d, bf, norm, pre, post, gates, seed=1, **given):
        self.B, self.n, self.d, self.t = mx.binding, n, d, BF if bf else F32
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(s, generator=g, device="cuda").to(self.t)
        self.mem = {k: rnd(n, d) for k in ("x", "u", "dh", "dy")}
        self.mem.update({k: rnd(d) for k in ("pre_weight", "pre_bias", "post_weight", "post_bias")}, gate=rnd(max(gates, 1), d))
        out = lambda *s, t=self.t: torch.full(s, 4096.0, device="cuda", dtype=t)
        self.mem.update({k: out(n, d) for k in ("h", "y", "dx", "du")}, stats=out(n, 4, t=F32), dgate=out(max(gates, 1), d))
        self.mem.update({k: out(d) for k in ("dpre_weight", "dpre_bias", "dpost_weight", "dpost_bias")})
        need = self.B.lib().mx_residual_norm_workspace_bytes(n, d, gates)
        self.mem["workspace"] = torch.full((need,), 0x7F, device="cuda", dtype=torch.uint8)      # NaN where it is read unwritten
        at = lambda *names: {k: self.mem[k].data_ptr() for k in names}
        self.a = self.B.ResidualNormArgs(rows=n, cols=d, ldx=d, ldu=d, ldh=d, ldy=d, x_dtype=int(bf), u_dtype=int(bf), norm=norm, pre=pre, post=post,
                                         param_dtype=int(bf), gate_dtype=int(bf), gate_rows=gates, ld_gate=d, residual_scale=1.25, branch_scale=0.7,
                                         eps=1e-6, **at("x", "u", "h", "stats", *(["y"] if pre else []), *(["gate"] if gates else [])))
        self.b = self.B.ResidualNormGrads(branch=1, lddh=d, lddy=d, lddx=d, lddu=d, workspace_bytes=need, **at("dh", "dx", "du", "workspace"))
        self.at = at

    def run(self, a=(), b=()):
        """Both passes with these arguments given as well; what came out of them."""
        for names, to in ((a, self.a), (b, self.b)):
            for k, v in self.at(*names).items():
                setattr(to, k, v)
        st = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
        assert self.B.lib().mx_residual_norm_fwd(ctypes.byref(self.a), st) == 0
        assert self.B.lib().mx_residual_norm_bwd(ctypes.byref(self.a), ctypes.byref(self.b), st) == 0
        return {k: self.mem[k].clone() for k in ("h", "y", "dx", "du", "dgate", "dpre_weight", "dpre_bias", "dpost_weight", "dpost_bias", "stats")}


@pytest.mark.parametrize("d", [5, 40, 41, 1001, 1024, 8200, 8203])
@pytest.mark.parametrize("norm", [0, 1])
def test_weights_of_a_norm_that_there_is_not(mx, d, norm):
    """Weights and biases that stand in the arguments without their norm, and an RMS norm's biases, change nothing."""
    for i, (pre, post) in enumerate(((1, 0), (0, 1), (0, 0), (1, 1))):
        for gates in (0, 1, 3):
            print("norms", pre, post, gates, flush=True)
            call = lambda: Call(mx, 6, d, bool(i % 2), norm, pre, post, gates, seed=i)
            wanted = (["dgate"] if gates else []) + (["dy", "dpre_weight"] if pre else []) + (["dpost_weight"] if post else [])
            own = (["pre_weight"] if pre else []) + (["post_weight"] if post else [])
            if norm == 1:
                own += (["pre_bias"] if pre else []) + (["post_bias"] if post else [])
            want = call().run(own, wanted)
            got = call().run(("pre_weight", "pre_bias", "post_weight", "post_bias"), wanted)
            for k in want:
                if k != "stats":
                    assert torch.equal(got[k], want[k]), (pre, post, gates, k)


@pytest.mark.parametrize("d", [5, 40, 41, 1001, 1024, 8200, 8203])
@pytest.mark.parametrize("norm", [0, 1])
@pytest.mark.parametrize("bf", [False, True])
def test_gradients_of_what_has_no_part_are_zero(mx, d, norm, bf):
    """Every gradient that is asked for is written: zeros where dy is NULL and where there is no such norm or bias."""
    params = ("pre_weight", "pre_bias", "post_weight", "post_bias")
    for pre, post, dy in ((1, 1, 0), (1, 1, 1), (1, 0, 1), (1, 0, 0), (0, 1, 0), (0, 0, 0)):
        for gates in (0, 1, 3):
            print("zeros", pre, post, dy, gates, flush=True)
            got = Call(mx, 6, d, bf, norm, pre, post, gates).run(params, ["d" + k for k in params] + (["dy"] if dy else []) + (["dgate"] if gates else []))
            for k, part in (("pre_weight", pre and dy), ("pre_bias", pre and dy and norm), ("post_weight", post), ("post_bias", post and norm)):
                r = got["d" + k]
                assert torch.isfinite(r).all() and not (r == 4096.0).any(), k
                assert part or not r.any(), (k, pre, post, dy, gates)
                assert not part or r.any(), (k, pre, post, dy, gates)
            assert not gates or (torch.isfinite(got["dgate"]).all() and not (got["dgate"] == 4096.0).any())


@pytest.mark.parametrize("ckpt", [False, True])
def test_saved_tensors_that_come_back_as_others(mx, ckpt):
    """A parameter, gate or matrix that saved-tensor hooks hand back with another type, size, shape or place is refused; one
    with other strides, or a copy, is taken."""
    n, d = 96, 64
    g = torch.Generator(device="cuda").manual_seed(31)
    x, u, p = make(g, n, d, BF, BF, BF, True, True, 3)
    leaves = {"x": x, "u": u, **p}
    for t in leaves.values():
        t.requires_grad_(True)
    dh, dy = (torch.randn((n, d), generator=g, device="cuda").to(BF) for _ in range(2))

    def step(name=None, change=None):
        mine = leaves[name].data_ptr() if name in leaves else None

        def pack(t):
            hit = t.data_ptr() == mine if mine else name == "h" and t.shape == x.shape and t.data_ptr() != u.data_ptr()
            seen.append(hit)
            return hit, t
        seen = []
        with torch.autograd.graph.saved_tensors_hooks(pack, lambda s: change(s[1]) if s[0] else s[1]):
            out = mx.residual_norm(x, u, **p, norm="layer", post=True, checkpoint=ckpt)
        assert name is None or sum(seen) == 1, name
        return torch.autograd.grad(out, list(leaves.values()), (dh, dy))
    want = step()
    spread = lambda t: torch.stack([t, t], -1).flatten(-2)[..., ::2]
    for name in ("pre_weight", "post_weight", "post_bias", "gate") + (() if ckpt else ("h", "u")):
        for same in (torch.clone, spread):
            assert all(torch.equal(a, b) for a, b in zip(step(name, same), want)), name
        other = [lambda t: t.float(), lambda t: t.half(), lambda t: t[..., :-1], lambda t: t.cpu(), lambda t: t.unsqueeze(0), lambda t: t.reshape(-1)[:1]]
        if name in ("gate", "h", "u"):
            other += [lambda t: t.t().contiguous(), lambda t: t[:1], lambda t: t.reshape(-1)]
        for i, change in enumerate(other):
            print("hook", name, i, flush=True)
            with pytest.raises((mx.MxError, TypeError)):
                step(name, change)


@pytest.mark.parametrize("d", [40, 41, 8200])
@pytest.mark.parametrize("norm", [0, 1])
def test_norm_alone_through_the_c_interface(mx, d, norm):
    """Without a block the post-norm's gradients are zeros too, and the others those of the norm."""
    n = 6
    call = Call(mx, n, d, False, norm, 1, 0, 0)
    call.a.u = call.a.h = call.b.dh = call.b.du = None
    call.b.branch = 0
    got = call.run(("pre_weight", "pre_bias"), ("dy", "dpre_weight", "dpre_bias", "dpost_weight", "dpost_bias"))
    assert not got["dpost_weight"].any() and not got["dpost_bias"].any()
    x, w, c = (call.mem[k].clone().requires_grad_(True) for k in ("x", "pre_weight", "pre_bias"))
    _, y = mx.residual_norm(x, pre_weight=w, pre_bias=c if norm else None, norm="layer" if norm else "rms")
    want = torch.autograd.grad(y, [x, w] + ([c] if norm else []), call.mem["dy"])
    # one scale of 1 in both: the residual's is not used without a block
    for k, t in zip(("dx", "dpre_weight", "dpre_bias"), want):
        assert torch.equal(got[k], t), k
    assert norm or not got["dpre_bias"].any()


def test_saved_input_of_a_norm_alone(mx):
    x = torch.randn((96, 64), device="cuda", requires_grad=True)
    for change, fits in ((torch.clone, True), (lambda t: t.t().contiguous(), False), (lambda t: t[:95], False), (lambda t: t.to(BF), False)):
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: change(t) if t.shape == x.shape else t):
            _, y = mx.residual_norm(x)
        if fits:
            torch.autograd.grad(y.sum(), x)
        else:
            with pytest.raises(mx.MxError):
                torch.autograd.grad(y.sum(), x)
