"""Operators between the linear layers on the GPU: values that are not finite, arguments that a norm does not read, results
that are zero.  Against the definitions in 64 bits (block_ref), with the bounds of test_gpu_block."""
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
