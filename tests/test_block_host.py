"""Operators between the linear layers, without a GPU: the 64-bit definitions that the GPU tests compare with are
checked against differences, and every call here is refused before anything is launched."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
import block_ref as ref  # noqa: E402


@pytest.fixture(scope="module")
def mx():
    import paper_2502_20853_amd as mx
    from paper_2502_20853_amd import build
    if build.is_stale():
        build.build()
    mx.binding.host()
    return mx


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("gates", [0, 1, 3, 6])
def test_gradients_of_the_definition_are_its_differences(layer, post, gates):
    g = torch.Generator().manual_seed(7 * layer + 3 * post + gates)
    n, d = 6, 5
    rnd = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)
    x, u, dh, dy = (rnd(n, d) for _ in range(4))
    p = {"pre_weight": 1 + 0.2 * rnd(d), "pre_bias": rnd(d), "post_weight": 1 + 0.2 * rnd(d), "post_bias": rnd(d), "gate": rnd(max(gates, 1), d)}
    if not gates:
        del p["gate"]
    if not layer:
        del p["pre_bias"], p["post_bias"]
    if not post:
        p = {k: v for k, v in p.items() if not k.startswith("post")}
    o = dict(layer=layer, post=post, rho=1.25, sigma=0.7, eps=1e-3)

    def loss(x, u, p):
        h = ref.forward_h(x, u, p, o)[0]
        y = ref.norm(h, layer, o["eps"], p["pre_weight"], p.get("pre_bias"))[0]
        return (h * dh).sum() + (y * dy).sum()

    h = ref.forward_h(x, u, p, o)[0]
    got = ref.backward((n, d), h, u, h, u, dh, dy, p, o)
    leaves = {"x": x, "u": u, **p}
    step = 1e-5
    for name, t in leaves.items():
        want = torch.zeros_like(t)
        for i in range(t.numel()):
            e = torch.zeros_like(t).view(-1)
            e[i] = step
            e = e.view_as(t)
            two = []
            for sign in (1, -1):
                moved = {k: (v + sign * e if k == name else v) for k, v in leaves.items()}
                two.append(loss(moved["x"], moved["u"], {k: moved[k] for k in p}))
            want.view(-1)[i] = (two[0] - two[1]) / (2 * step)
        # central differences: third derivatives times step^2, and 2^-53 of the loss over the step
        assert torch.allclose(got[name][0].view_as(want), want, rtol=1e-6, atol=1e-7), name


@pytest.mark.parametrize("kind", ["gelu", "silu"])
def test_slope_of_the_definition_is_its_difference(kind):
    x = torch.linspace(-9, 9, 1001, dtype=torch.float64)
    a, b = ref.act(kind, x + 1e-5)[0], ref.act(kind, x - 1e-5)[0]
    assert torch.allclose(ref.act(kind, x)[1], (a - b) / 2e-5, rtol=0, atol=1e-9)


def test_eight_bit_definition():
    x = torch.tensor([[448.0, 1.0, 0.0, -0.4]])
    assert torch.equal(ref.eight_bits(x)[0].float(), torch.tensor([[448.0, 1.0, 0.0, -0.40625]])) and ref.eight_bits(x)[1].item() == 127
    assert ref.eight_bits(torch.tensor([[448.5]]))[1].item() == 128
    assert ref.eight_bits(torch.zeros(1, 40))[1].tolist() == [[0, 0]]
    # as torch's own conversion, where the scale is 1
    y = torch.linspace(-448, 448, 4097)
    y = torch.cat([y, torch.full((31,), 448.0)]).view(-1, 32)
    y[:, 0] = 448.0
    assert torch.equal(ref.eight_bits(y)[0].float(), y.to(torch.float8_e4m3fn).float())


def refused(mx, code, call, *args, **kw):
    with pytest.raises(mx.MxError) as e:
        call(*args, **kw)
    assert e.value.code == code, e.value


def test_residual_norm_refusals(mx):
    B = mx.binding
    x, w = torch.zeros(6, 64), torch.ones(64)
    bf = torch.bfloat16
    for bad in (dict(norm="batch"), dict(u=torch.zeros(6, 32)), dict(pre_weight=torch.ones(63)), dict(pre_weight=torch.ones(1, 64)),
                dict(pre_bias=w), dict(post_weight=w), dict(gate=w), dict(residual_scale=2.0), dict(post=True), dict(pre=False),
                dict(u=x, post_bias=w, post=True), dict(u=x, gate=torch.ones(32)), dict(u=x, gate=torch.ones(4, 64)),
                dict(u=x, pre=False, packed=True), dict(u=x, pre=False, pre_weight=w)):
        with pytest.raises(ValueError):
            mx.residual_norm(x, **bad)
    with pytest.raises(ValueError):                                       # a row for each position: not one for a run of rows
        mx.residual_norm(torch.zeros(2, 3, 64), torch.zeros(2, 3, 64), gate=torch.ones(3, 64))
    with pytest.raises(ValueError):
        mx.residual_norm(torch.zeros(2, 3, 64), torch.zeros(2, 3, 64), gate=torch.ones(1, 3, 64))
    for bad in (dict(x=x.half()), dict(x=x, u=x.double()), dict(x=x, pre_weight=w.half()), dict(x=x, u=x, gate=w.half()),
                dict(x=x, u=x, post=True, pre_weight=w, post_weight=w.to(bf))):
        with pytest.raises(TypeError):
            mx.residual_norm(**bad)
    refused(mx, B.MX_ERR_SHAPE, mx.residual_norm, torch.zeros(0, 64))
    refused(mx, B.MX_ERR_SHAPE, mx.residual_norm, torch.zeros(4, 0))
    refused(mx, B.MX_ERR_SHAPE, mx.residual_norm, torch.zeros(1, 16385))
    refused(mx, B.MX_ERR_SHAPE, mx.residual_norm, torch.zeros(4, 40), packed=True)
    refused(mx, B.MX_ERR_DTYPE, mx.residual_norm, x.to(bf), x)
    refused(mx, B.MX_ERR_MODE, mx.residual_norm, x, scale_mode=3)
    for eps in (0.0, -1e-6, float("nan"), float("inf"), 1e-45):
        refused(mx, B.MX_ERR_MODE, mx.residual_norm, x, eps=eps)
    for scale in (float("nan"), float("inf")):
        refused(mx, B.MX_ERR_MODE, mx.residual_norm, x, x, residual_scale=scale)
        refused(mx, B.MX_ERR_MODE, mx.residual_norm, x, x, branch_scale=scale)
    with pytest.raises(RuntimeError, match="GPU"):
        mx.residual_norm(x, x)
    with pytest.raises(ValueError):
        mx.MxResidualNorm(64, norm="x", device="cpu")
    with pytest.raises(ValueError):
        mx.MxResidualNorm(64, gate=0.5, device="cpu")(x, x, gate=w)


def test_activation_and_checkpoint_refusals(mx):
    B = mx.binding
    p = torch.zeros(4, 64)
    with pytest.raises(ValueError):
        mx.activation(p, "relu")
    with pytest.raises(ValueError):
        mx.MxActivation("tanh")
    with pytest.raises(ValueError):
        mx.activation(torch.zeros(4, 63), gated=True)
    with pytest.raises(TypeError):
        mx.activation(p.half())
    refused(mx, B.MX_ERR_SHAPE, mx.activation, torch.zeros(0, 64))
    refused(mx, B.MX_ERR_SHAPE, mx.activation, torch.zeros(4, 40), packed=True)
    refused(mx, B.MX_ERR_SHAPE, mx.activation, torch.zeros(4, 96), gated=True, packed=True)
    refused(mx, B.MX_ERR_MODE, mx.activation, p, scale_mode=-1)
    with pytest.raises(RuntimeError, match="GPU"):
        mx.activation(p)
    with pytest.raises(TypeError):
        mx.mx_checkpoint_pack(p.int())
    refused(mx, B.MX_ERR_SHAPE, mx.mx_checkpoint_pack, torch.zeros(3, 0))
    with pytest.raises(RuntimeError, match="GPU"):
        mx.mx_checkpoint_pack(p)
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)
    with pytest.raises(TypeError):
        mx.mx_checkpoint_unpack(u8(4, 64), u8(4, 2), 64, torch.float16)
    for codes, scales, cols in ((u8(4, 64), u8(4, 2), 65), (u8(4, 64), u8(4, 1), 64), (u8(4, 64).int(), u8(4, 2), 64)):
        with pytest.raises(ValueError):
            mx.mx_checkpoint_unpack(codes, scales, cols)
    with pytest.raises(ValueError):
        mx.mx_checkpoint_unpack(u8(4, 64), u8(4, 2), 64, out=torch.zeros(4, 64, dtype=torch.bfloat16))
    with pytest.raises(RuntimeError, match="GPU"):
        mx.mx_checkpoint_unpack(u8(4, 64), u8(4, 2), 64)


def test_forward_mode_is_refused(mx):
    import torch.autograd.forward_ad as fwAD
    with fwAD.dual_level():
        x = fwAD.make_dual(torch.zeros(4, 64), torch.ones(4, 64))
        for call in (mx.residual_norm, mx.activation):
            with pytest.raises(NotImplementedError):
                call(x)


FAKE = 0x7F0000000000          # never dereferenced: every call below fails validation first


def test_c_interface_refusals(mx):
    B, L = mx.binding, mx.binding.lib()
    P = ctypes.c_void_p

    def pack(fn="mx_checkpoint_pack", values=FAKE, dtype=1, rows=4, cols=64, ld=64, codes=FAKE, scales=FAKE):
        if fn == "mx_checkpoint_pack":
            return L.mx_checkpoint_pack(P(values), dtype, rows, cols, ld, P(codes), P(scales), P(0))
        return L.mx_checkpoint_unpack(P(codes), P(scales), rows, cols, P(values), dtype, ld, P(0))
    for fn in ("mx_checkpoint_pack", "mx_checkpoint_unpack"):
        assert pack(fn, values=0) == -1 and pack(fn, codes=0) == -1 and pack(fn, scales=0) == -1
        assert pack(fn, dtype=2) == -3
        assert pack(fn, rows=0) == -2 and pack(fn, cols=0) == -2 and pack(fn, ld=63) == -2 and pack(fn, rows=1 << 30, cols=64) == -2
        assert pack(fn, values=FAKE + 1) == -5 and pack(fn, codes=FAKE + 4) == -5 and pack(fn, dtype=0, values=FAKE + 2) == -5

    def fwd(**kw):
        a = B.ResidualNormArgs(rows=4, cols=64, x=FAKE, u=FAKE, h=FAKE, y=FAKE, ldx=64, ldu=64, ldh=64, ldy=64, x_dtype=1, u_dtype=1,
                               pre=1, post=1, gate_rows=1, ld_gate=64, residual_scale=1.0, branch_scale=1.0, eps=1e-6)
        for k, v in kw.items():
            setattr(a, k, v)
        return L.mx_residual_norm_fwd(ctypes.byref(a), P(0))
    assert L.mx_residual_norm_fwd(P(0), P(0)) == -1
    assert fwd(x=0) == -1 and fwd(h=0) == -1 and fwd(y=0) == -1 and fwd(u=0) == -1
    assert fwd(y_codes=FAKE) == -1 and fwd(h8=FAKE) == -1 and fwd(u8_scales=FAKE) == -1
    assert fwd(u=0, h=0) == -4 and fwd(u=0, h=0, post=0, gate=FAKE) == -4                 # no branch to norm or gate
    assert fwd(y_codes=FAKE, y_scales=FAKE) == -4 and fwd(pre=0) == -4                    # one y, or none
    assert fwd(pre=2) == -4 and fwd(post=-1) == -4 and fwd(norm=2) == -4 and fwd(eps=0.0) == -4
    assert fwd(y=0, y_codes=FAKE, y_scales=FAKE, scale_mode=2) == -4
    assert fwd(x_dtype=2) == -3 and fwd(u_dtype=5) == -3 and fwd(param_dtype=-1) == -3 and fwd(u_dtype=0) == -3 and fwd(gate=FAKE, gate_dtype=9) == -3
    assert fwd(rows=0) == -2 and fwd(cols=0) == -2 and fwd(cols=16385, ldx=16385, ldu=16385, ldh=16385, ldy=16385) == -2
    assert fwd(ldx=63) == -2 and fwd(ldh=0) == -2 and fwd(gate=FAKE, gate_rows=3) == -2 and fwd(gate=FAKE, gate_rows=0) == -2
    assert fwd(gate=FAKE, gate_rows=2, ld_gate=63) == -2
    assert fwd(cols=40, y=0, y_codes=FAKE, y_scales=FAKE) == -2
    assert fwd(x=FAKE + 1) == -5 and fwd(h8=FAKE + 4, h8_scales=FAKE) == -5 and fwd(stats=FAKE + 8) == -5
    assert fwd(pre_weight=FAKE + 2) == -5 and fwd(y=0, y_codes=FAKE + 8, y_scales=FAKE) == -5

    need = L.mx_residual_norm_workspace_bytes(4, 64, 0)
    assert need > 0 and L.mx_residual_norm_workspace_bytes(0, 64, 0) == 0 and L.mx_residual_norm_workspace_bytes(4, 64, 5) == 0

    def bwd(**kw):
        a = B.ResidualNormArgs(rows=4, cols=64, x=FAKE, u=FAKE, h=FAKE, ldx=64, ldu=64, ldh=64, x_dtype=1, u_dtype=1, pre=1, post=1,
                               residual_scale=1.0, branch_scale=1.0, eps=1e-6, stats=FAKE)
        d = B.ResidualNormGrads(branch=1, dh=FAKE, dy=FAKE, dx=FAKE, du=FAKE, lddh=64, lddy=64, lddx=64, lddu=64, workspace=FAKE, workspace_bytes=need)
        for k, v in kw.items():
            setattr(d if k in dict(B.ResidualNormGrads._fields_) else a, k, v)
        return L.mx_residual_norm_bwd(ctypes.byref(a), ctypes.byref(d), P(0))
    assert L.mx_residual_norm_bwd(P(0), P(0), P(0)) == -1
    assert bwd(dh=0, dy=0) == -1 and bwd(stats=0) == -1 and bwd(h=0) == -1 and bwd(u=0) == -1 and bwd(h8=FAKE) == -1 and bwd(dgate=FAKE) == -1
    assert bwd(h8=FAKE, h8_scales=FAKE) == -1                                             # then u's checkpoint is needed too
    assert bwd(branch=2) == -4 and bwd(pre=0) == -4 and bwd(branch=0, post=0) == -4
    assert bwd(workspace=0) == -6 and bwd(workspace_bytes=need - 1) == -6
    assert bwd(lddy=60) == -2 and bwd(lddx=1) == -2 and bwd(workspace=FAKE + 8) == -5 and bwd(dy=FAKE + 1) == -5 and bwd(dpre_weight=FAKE + 2) == -5

    def act(fn="fwd", p=FAKE, dtype=1, rows=4, cols=64, ldp=128, kind=0, gated=1, a=FAKE, lda=64, ac=0, as_=0, mode=0, p8=0, p8s=0, dp=FAKE):
        if fn == "fwd":
            return L.mx_activation_fwd(P(p), dtype, rows, cols, ldp, kind, gated, P(a), lda, P(ac), P(as_), mode, P(p8), P(p8s), P(0))
        return L.mx_activation_bwd(P(p), P(p8), P(p8s), dtype, rows, cols, ldp, kind, gated, P(a), lda, P(dp), 128, P(0))
    for fn in ("fwd", "bwd"):
        assert act(fn, p=0) == -1 and act(fn, a=0) == -1 and act(fn, p8=FAKE) == -1
        assert act(fn, dtype=4) == -3 and act(fn, kind=2) == -4 and act(fn, gated=2) == -4
        assert act(fn, rows=0) == -2 and act(fn, cols=0) == -2 and act(fn, ldp=127) == -2 and act(fn, lda=63) == -2
        assert act(fn, p=FAKE + 1) == -5 and act(fn, a=FAKE + 1) == -5 and act(fn, p8=FAKE + 4, p8s=FAKE) == -5
    assert act("bwd", dp=0) == -1
    assert act(ac=FAKE) == -1 and act(ac=FAKE, as_=FAKE) == -4 and act(a=0, ac=FAKE, as_=FAKE, mode=5) == -4
    assert act(a=0, ac=FAKE + 8, as_=FAKE) == -5 and act(a=0, ac=FAKE, as_=FAKE, cols=48) == -2


def test_workspace_of_sizes_that_no_call_takes(mx):
    need = mx.binding.lib().mx_residual_norm_workspace_bytes
    for rows, cols in ((1, 16385), (1, 1 << 20), (1, 1 << 40), (1 << 62, 64), (1 << 30, 64), ((1 << 63) - 1, 1), (-1, 64), (4, -64)):
        assert need(rows, cols, 0) == 0 and need(rows, cols, 1) == 0, (rows, cols)
    most = (1 << 35) - (1 << 19)                                          # elements of a call
    for cols in (32, 16384):
        assert need(most // cols + 1, cols, 0) == 0
    for rows, cols in ((1, 1), (1, 16384), (most // 16384, 16384), (most // 32, 32)):
        for gates in (0, 1, rows):
            assert need(rows, cols, gates) > 0, (rows, cols, gates)


def test_checkpoint_of_scattered_values_on_a_given_stream(mx):
    """They would be gathered on the current stream."""
    with pytest.raises(ValueError, match="stream"):
        mx.mx_checkpoint_pack(torch.zeros(64, 4).t(), stream=1)
    with pytest.raises(ValueError, match="stream"):
        mx.mx_checkpoint_pack(torch.zeros(2, 4, 128)[:, :, :64], stream=1)
    for values in (torch.zeros(4, 64), torch.zeros(4, 128)[:, :64], torch.zeros(2, 4, 64)):
        with pytest.raises(RuntimeError, match="GPU"):
            mx.mx_checkpoint_pack(values, stream=1)


def test_module_without_a_branch_refuses_what_needs_one(mx):
    """A gate, or a module without a pre-norm, has no part in the norm of x alone."""
    x, w = torch.zeros(6, 64), torch.ones(64)
    for kw in (dict(), dict(norm="layer"), dict(post=True), dict(gate=0.5)):
        with pytest.raises(ValueError):
            mx.MxResidualNorm(64, device="cpu", **kw)(x, gate=w)
        with pytest.raises(ValueError):
            mx.MxResidualNorm(64, device="cpu", pre=False, **kw)(x)
        with pytest.raises(ValueError):
            mx.MxResidualNorm(64, device="cpu", pre=False, **kw)(x, packed=True)
        with pytest.raises(RuntimeError, match="GPU"):                    # these are calls
            mx.MxResidualNorm(64, device="cpu", **kw)(x)
        with pytest.raises(RuntimeError, match="GPU"):
            mx.MxResidualNorm(64, device="cpu", pre=False, **kw)(x, x)
