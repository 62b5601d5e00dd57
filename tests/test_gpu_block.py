"""Operators between the linear layers on the GPU against their definitions in 64 bits (block_ref), with bounds that count
the roundings of FP32 arithmetic."""
import pytest

torch = pytest.importorskip("torch")
import block_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
EPS = 1e-6


@pytest.fixture(scope="module")
def mx():
    import paper_2502_20853_amd as mx
    mx.binding.host()
    return mx


def check(got, value, scale, ops, what):
    t = got.dtype
    g = got.detach().cpu().double()
    assert g.shape == value.shape, (what, g.shape, value.shape)
    assert torch.isfinite(g).all(), what
    err = ops * ref.EPS * scale
    # the last rounding works on the FP32 result; below the smallest normal value steps stay 2^-133 (bf16) or 2^-149
    tol = err + ref.HALF_STEP[t] * (value.abs() + err) + 2.0 ** -133
    worst = ((g - value).abs() / tol.clamp_min(1e-300)).max().item()
    assert worst <= 1.0, "%s: %.3g of the bound" % (what, worst)


def make(g, n, d, xt, ut, pt, layer, post, gates, affine=True):
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")
    x = rnd(n, d)
    x[:, torch.randperm(d, generator=g, device="cuda")[: max(1, d // 100)]] *= 20.0
    u = rnd(n, d) * 0.7 + 0.1
    p = {}
    if affine:
        p["pre_weight"] = 1 + 0.2 * rnd(d)
        if layer:
            p["pre_bias"] = 0.3 * rnd(d)
        if post:
            p["post_weight"] = 1 + 0.2 * rnd(d)
            if layer:
                p["post_bias"] = 0.3 * rnd(d)
    if gates:
        p["gate"] = 0.5 + 0.25 * rnd(gates, d)
    return x.to(xt), u.to(ut), {k: v.to(pt) for k, v in p.items()}


def f64(t):
    return t.detach().cpu().double()


# roundings on the way to a value, relative to its terms: sums in a row take 8 to 16 additions in a lane, 6 across a wave, 4
# across waves, in the mean and in the squares; the products, quotients and roots around them about ten more
FORWARD_OPS, BACKWARD_OPS = 48, 128


def run_case(mx, n, d, xt, ut, pt, layer, post, gates, ckpt, seed, rho=1.25, sigma=0.7, use=("h", "y"), affine=True, branch=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, u, p = make(g, n, d, xt, ut, pt, layer, post, gates, affine)
    dh = (torch.randn((n, d), generator=g, device="cuda") * 1e-2).to(xt)
    dy = (torch.randn((n, d), generator=g, device="cuda") * 1e-2).to(ut)
    if not branch:
        u, rho, sigma, p = None, 1.0, 1.0, {k: v for k, v in p.items() if k.startswith("pre")}
    o = dict(layer=layer, post=post, rho=rho, sigma=sigma, eps=EPS)
    leaves = {"x": x, **({"u": u} if branch else {}), **p}
    for t in leaves.values():
        t.requires_grad_(True)
    kw = dict(norm="layer" if layer else "rms", eps=EPS, checkpoint=ckpt)
    if branch:
        kw.update(post=post, residual_scale=rho, branch_scale=sigma)
    h, y = mx.residual_norm(x, u, **p, **kw)
    with torch.no_grad():
        h2, y2 = mx.residual_norm(x, u, **p, **kw)
    assert torch.equal(h, h2) and torch.equal(y, y2)                      # keeping something changes no result
    x64, u64, p64 = f64(x), f64(u) if branch else None, {k: f64(v) for k, v in p.items()}
    if branch:
        assert h.dtype == xt and y.dtype == ut
        check(h, *ref.forward_h(x64, u64, p64, o), FORWARD_OPS, "h")
    else:
        assert h is x
    h64 = f64(h)
    check(y, *ref.norm(h64, layer, EPS, p64.get("pre_weight"), p64.get("pre_bias")), FORWARD_OPS, "y")

    outs = [(t, gr) for k, t, gr in (("h", h, dh), ("y", y, dy)) if k in use and (branch or k == "y")]
    grads = torch.autograd.grad([t for t, _ in outs], list(leaves.values()), [gr for _, gr in outs], allow_unused=True)
    again = mx.residual_norm(x, u, **p, **kw)
    outs2 = [(t, gr) for k, t, gr in (("h", again[0], dh), ("y", again[1], dy)) if k in use and (branch or k == "y")]
    grads2 = torch.autograd.grad([t for t, _ in outs2], list(leaves.values()), [gr for _, gr in outs2], allow_unused=True)
    h_kept, u_kept = (ref.eight_bits(f64(h))[0], ref.eight_bits(u64)[0] if branch else None) if ckpt else (h64, u64)
    dh64 = f64(dh) if "h" in use and branch else torch.zeros((n, d), dtype=torch.float64)
    want = ref.backward((n, d), h64, u64, h_kept, u_kept, dh64, f64(dy) if "y" in use else None, p64, o)
    for (name, leaf), got, rep in zip(leaves.items(), grads, grads2):
        if name not in want:
            assert got is None, name
            continue
        assert got.dtype == leaf.dtype and got.shape == leaf.shape
        assert torch.equal(got, rep), name + " does not repeat"
        value, scale, rows = want[name]
        check(got, value.view(leaf.shape), scale.view(leaf.shape), BACKWARD_OPS + rows, "d " + name)


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("ckpt", [False, True])
@pytest.mark.parametrize("types", [(BF, BF, F32), (F32, BF, BF), (F32, F32, F32), (BF, BF, BF)])
def test_residual_norm(mx, layer, post, ckpt, types):
    print("case", layer, post, ckpt, types, flush=True)
    run_case(mx, 70, 96, *types, layer, post, 1, ckpt, 1)
    run_case(mx, 33, 768, *types, layer, post, 0, ckpt, 2)


@pytest.mark.parametrize("d", [1, 2, 3, 7, 8, 9, 31, 32, 33, 63, 65, 127, 250, 500, 512, 513, 1001, 1024, 1537, 4096, 4099, 8192, 8200, 16383, 16384])
@pytest.mark.parametrize("n", [1, 5])
def test_residual_norm_widths(mx, d, n):
    for i, types in enumerate([(BF, BF, BF), (F32, BF, F32), (F32, F32, F32)]):
        layer, ckpt = (d + i) % 2 == 0, (n + i) % 2 == 0
        print("width", d, n, types, layer, ckpt, flush=True)
        run_case(mx, n, d, *types, layer, True, 1, ckpt, 10 + i)


@pytest.mark.parametrize("d", [33, 1001, 4099, 12001])
def test_odd_rows_of_every_kind(mx, d):
    """Rows of no whole vectors, with and without a post-norm, a gate, gate rows, 8-bit checkpoints."""
    i = 0
    for layer in (False, True):
        for post in (False, True):
            for gates in (0, 1, 3):
                for ckpt in (False, True):
                    i += 1
                    print("odd", d, layer, post, gates, ckpt, flush=True)
                    run_case(mx, 9, d, *[(BF, BF, BF), (F32, BF, F32), (F32, F32, F32)][i % 3], layer, post, gates, ckpt, 40 + i)


@pytest.mark.parametrize("d", [768, 2048, 4096, 8192, 16384])
def test_whole_rows_of_every_kind(mx, d):
    i = 0
    for layer in (False, True):
        for post in (False, True):
            for gates in (0, 1, 3):
                for ckpt in (False, True):
                    i += 1
                    print("whole", d, layer, post, gates, ckpt, flush=True)
                    run_case(mx, 9, d, *[(BF, BF, BF), (F32, BF, F32), (F32, F32, F32)][i % 3], layer, post, gates, ckpt, 70 + i)


@pytest.mark.parametrize("n,d,gates", [(12, 40, 12), (12, 40, 4), (600, 72, 2), (600, 72, 300), (1970, 192, 10), (4096, 64, 4096), (1, 64, 1),
                                       (1200, 33, 600), (5000, 520, 25), (3000, 1100, 1500)])
def test_gate_rows(mx, n, d, gates):
    for i, (layer, post, ckpt) in enumerate([(False, True, True), (True, False, False), (True, True, True)]):
        print("gates", n, d, gates, i, flush=True)
        run_case(mx, n, d, BF if i else F32, BF, F32 if i == 1 else BF, layer, post, gates, ckpt, 20 + i)


@pytest.mark.parametrize("n,d", [(257, 192), (2048, 64), (4097, 256), (3000, 768), (1030, 4096), (700, 8192), (300, 10000)])
def test_residual_norm_many_rows(mx, n, d):
    for layer, ckpt in ((False, True), (True, False)):
        print("rows", n, d, layer, ckpt, flush=True)
        run_case(mx, n, d, BF, BF, F32, layer, True, 1, ckpt, 3)


@pytest.mark.parametrize("n,d,gates", [(600, 8192, 2), (600, 8192, 600), (300, 8200, 300), (300, 8200, 3), (300, 9001, 5), (130, 16384, 130)])
def test_wide_rows_with_gate_rows(mx, n, d, gates):
    for i, (layer, post, ckpt) in enumerate([(False, True, True), (True, True, False), (False, False, False)]):
        print("wide gates", n, d, gates, i, flush=True)
        run_case(mx, n, d, F32 if i == 1 else BF, BF, BF, layer, post, gates, ckpt, 90 + i)


@pytest.mark.parametrize("d", [8200, 10000])
def test_wide_rows_whose_inputs_alone_want_gradients(mx, d):
    g = torch.Generator(device="cuda").manual_seed(95)
    x, u, p = make(g, 70, d, BF, BF, BF, False, True, 5)
    gr = torch.randn((2, 70, d), generator=g, device="cuda").to(BF)
    every = [t.requires_grad_(True) for t in (x, u, *p.values())]
    want = torch.autograd.grad(mx.residual_norm(x, u, **p, post=True), every, (gr[0], gr[1]))
    plain = {k: v.detach() for k, v in p.items()}
    got = torch.autograd.grad(mx.residual_norm(x, u, **plain, post=True), (x, u), (gr[0], gr[1]))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    (gate,) = torch.autograd.grad(mx.residual_norm(x, u, **{**plain, "gate": p["gate"]}, post=True), (p["gate"],), (gr[0], gr[1]))
    assert torch.equal(gate, want[-1])


@pytest.mark.parametrize("use", [("h",), ("y",)])
@pytest.mark.parametrize("ckpt", [False, True])
def test_one_gradient_is_missing(mx, use, ckpt):
    run_case(mx, 40, 200, BF, BF, F32, True, True, 1, ckpt, 4, use=use)
    run_case(mx, 40, 200, F32, F32, F32, False, False, 0, ckpt, 4, use=use)


@pytest.mark.parametrize("ckpt", [False, True])
def test_norm_alone_and_without_parameters(mx, ckpt):
    run_case(mx, 40, 200, BF, BF, F32, True, False, 0, ckpt, 5, use=("y",), branch=False)
    run_case(mx, 40, 200, F32, F32, F32, False, False, 0, ckpt, 5, use=("y",), branch=False)
    run_case(mx, 40, 200, BF, BF, F32, True, True, 1, ckpt, 5, affine=False)


def test_without_pre_norm(mx):
    g = torch.Generator(device="cuda").manual_seed(6)
    for ckpt in (False, True):
        x, u, p = make(g, 50, 130, BF, BF, BF, False, True, 1)
        del p["pre_weight"]
        leaves = [t.requires_grad_(True) for t in (x, u, *p.values())]
        h, y = mx.residual_norm(x, u, **p, pre=False, post=True, checkpoint=ckpt)
        assert y is None
        dh = torch.randn((50, 130), generator=g, device="cuda").to(BF)
        grads = torch.autograd.grad(h, leaves, dh)
        o = dict(layer=False, post=True, rho=1.0, sigma=1.0, eps=1e-6)
        p64 = {k: f64(v) for k, v in p.items()}
        check(h, *ref.forward_h(f64(x), f64(u), p64, o), FORWARD_OPS, "h")
        u_kept = ref.eight_bits(f64(u))[0] if ckpt else f64(u)
        want = ref.backward((50, 130), f64(h), f64(u), None, u_kept, f64(dh), None, p64, o)
        for name, leaf, got in zip(("x", "u", *p), leaves, grads):
            check(got, want[name][0].view(leaf.shape), want[name][1].view(leaf.shape), BACKWARD_OPS + want[name][2], name)


def test_only_what_is_asked_for(mx):
    """Any subset of the inputs may want a gradient; the others get none and the result is the same."""
    g = torch.Generator(device="cuda").manual_seed(7)
    x, u, p = make(g, 64, 160, BF, BF, F32, True, True, 4)
    dh, dy = (torch.randn((64, 160), generator=g, device="cuda").to(BF) for _ in range(2))
    names = ["x", "u", *p]
    for ckpt in (False, True):
        full = None
        for wanted in [names] + [[k] for k in names] + [["u", "gate"], ["x", "post_bias"]]:
            leaves = {k: t.detach().clone().requires_grad_(k in wanted) for k, t in {"x": x, "u": u, **p}.items()}
            h, y = mx.residual_norm(leaves["x"], leaves["u"], **{k: leaves[k] for k in p}, norm="layer", post=True, checkpoint=ckpt)
            torch.autograd.backward((h, y), (dh, dy))
            got = {k: leaves[k].grad for k in names}
            assert all((got[k] is not None) == (k in wanted) for k in names)
            full = full or got
            assert all(torch.equal(got[k], full[k]) for k in wanted)


def test_shapes_strides_and_gate_forms(mx):
    g = torch.Generator(device="cuda").manual_seed(8)
    B, T, D = 3, 7, 88
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda").to(BF)
    x, u, w = rnd(B, T, D), rnd(B, T, D), rnd(D)
    plain = lambda x, u, gate: mx.residual_norm(x.reshape(-1, D).contiguous(), u.reshape(-1, D).contiguous(), pre_weight=w, gate=gate)
    for gate, rows in ((rnd(D), 1), (rnd(1, 1, D), 1), (rnd(B, 1, D), B), (rnd(B, T, D), B * T), (rnd(B, 6 * D)[:, D:2 * D].unsqueeze(1), B)):
        want = plain(x, u, gate.reshape(-1, D))
        got = mx.residual_norm(x, u, pre_weight=w, gate=gate)
        assert got[0].shape == (B, T, D) and all(torch.equal(a.reshape(-1, D), b) for a, b in zip(got, want)), rows
    # column slices, odd strides and addresses, transposed and expanded tensors
    want = plain(x, u, w)
    flat = lambda t: t.reshape(-1, D)
    wide = torch.zeros((B * T, 2 * D + 3), device="cuda", dtype=BF)
    wide[:, 3:3 + D], wide[:, 3 + D:] = flat(x), flat(u)
    for xs, us in ((wide[:, 3:3 + D], wide[:, 3 + D:]), (flat(x).t().contiguous().t(), flat(u)), (flat(x), flat(u).t().contiguous().t())):
        got = mx.residual_norm(xs, us, pre_weight=w, gate=w)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    one = x[:1, :1].reshape(1, D).expand(5, D)
    got = mx.residual_norm(one, one, pre_weight=w, gate=w)
    want = mx.residual_norm(one.contiguous(), one.contiguous(), pre_weight=w, gate=w)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # a vector is one row
    got = mx.residual_norm(x[0, 0], u[0, 0], pre_weight=w, gate=w)
    want = mx.residual_norm(x[0, :1], u[0, :1], pre_weight=w, gate=w)
    assert got[0].shape == (D,) and all(torch.equal(a, b[0]) for a, b in zip(got, want))
    # gradients of strided inputs arrive in the inputs' shapes
    xs, us = x.transpose(0, 1).detach().requires_grad_(True), wide[:, 3 + D:].reshape(B, T, D).transpose(0, 1).detach().requires_grad_(True)
    h, y = mx.residual_norm(xs, us, pre_weight=w, checkpoint=True)
    gx, gu = torch.autograd.grad(h.float().sum() + y.float().sum(), (xs, us))
    assert gx.shape == xs.shape and gu.shape == us.shape
    # outputs' gradients that are expanded, as a sum gives them, or transposed
    h, y = mx.residual_norm(xs, us, pre_weight=w, checkpoint=True)
    again = torch.autograd.grad((h, y), (xs, us), (torch.ones_like(h), torch.ones((), device="cuda", dtype=BF).expand(y.shape)))
    assert torch.equal(gx, again[0]) and torch.equal(gu, again[1])


def test_rows_are_independent(mx):
    """A row of zeros, infinities or NaN changes no other row; a row of zeros has finite results."""
    g = torch.Generator(device="cuda").manual_seed(9)
    for d in (48, 600):
        x, u, p = make(g, 9, d, BF, BF, BF, True, True, 1)
        h0, y0 = mx.residual_norm(x, u, **p, norm="layer", post=True)
        x[4], u[4] = 0, 0
        u[2, 5], x[7, 3], x[6, 1] = float("inf"), float("nan"), float("-inf")
        for t in (x, u):
            t.requires_grad_(True)
        h, y = mx.residual_norm(x, u, **p, norm="layer", post=True, checkpoint=True)
        rest = [0, 1, 3, 5, 8]
        assert torch.equal(h[rest], h0[rest]) and torch.equal(y[rest], y0[rest])
        assert torch.isfinite(h[4]).all() and torch.isfinite(y[4]).all()
        gx, gu = torch.autograd.grad((h, y), (x, u), (torch.ones_like(h), torch.ones_like(y)))
        assert torch.isfinite(gx[rest + [4]]).all() and torch.isfinite(gu[rest + [4]]).all()
        assert not torch.isfinite(gu[2]).all() and not torch.isfinite(gx[7]).all()


@pytest.mark.parametrize("floor", [False, True])
@pytest.mark.parametrize("n,d", [(1, 32), (5, 64), (33, 768), (3, 4096), (2, 16384), (700, 224)])
def test_packed_output(mx, n, d, floor):
    mode = mx.SCALE_FLOOR if floor else mx.SCALE_TRUNCFREE
    g = torch.Generator(device="cuda").manual_seed(11)
    for layer, xt, ut in ((False, BF, BF), (True, F32, F32)):
        x, u, p = make(g, n, d, xt, ut, F32, layer, True, 1)
        kw = dict(norm="layer" if layer else "rms", post=True)
        h, (codes, scales) = mx.residual_norm(x, u, **p, **kw, packed=True, scale_mode=mode)
        h2, y = mx.residual_norm(x.float(), u.float(), **p, **kw) if xt == F32 else (h, None)
        assert torch.equal(h, h2) and codes.shape == (n, d // 2) and scales.shape == (n, d // 32)
        if y is not None:                                 # FP32 values: the codes are those of the row quantizer, byte for byte
            want = mx.mx_quantize(y, scale_mode=mode)
            assert torch.equal(codes, want[0]) and torch.equal(scales, want[1])
        else:
            check_codes(mx, codes, scales, *ref.norm(f64(h), layer, EPS, f64(p["pre_weight"]), None), floor)


def check_codes(mx, codes, scales, value, scale, floor):
    """Every code is one that some value within the bound has, under a scale that some maximum within it has."""
    err = FORWARD_OPS * ref.EPS * scale
    n, d = value.shape
    codes = torch.stack([codes.cpu() & 15, codes.cpu() >> 4], -1).view(n, d)
    same = 0
    lo, slo = ref.four_bits(value - err, floor)
    hi, shi = ref.four_bits(value + err, floor)
    mid, smid = ref.four_bits(value, floor)
    got_s = scales.cpu()
    top = value.abs().view(n, -1, 32).amax(-1)
    top_err = err.view(n, -1, 32).amax(-1)
    a, b = (ref.four_bits((top + sign * top_err).unsqueeze(-1).expand(-1, -1, 32).reshape(n, d), floor)[1] for sign in (-1, 1))
    assert ((got_s == a) | (got_s == b)).all()
    agree = (got_s == smid).repeat_interleave(32, 1)
    fits = (codes == lo) | (codes == hi) | (codes == mid)
    near = (slo != shi).repeat_interleave(32, 1)
    assert (fits | ~agree | near).all()
    assert ((codes == mid) & agree).double().mean() > 0.999


def test_packed_goes_into_the_product(mx):
    """norm -> MXFP4 codes -> projection, and activation -> codes -> projection, as a serving program runs them."""
    g = torch.Generator(device="cuda").manual_seed(12)
    n, d, f = 5, 128, 256
    x, u, p = make(g, n, d, BF, BF, F32, False, True, 0)
    w1 = mx.mx_quantize(torch.randn((2 * f, d), generator=g, device="cuda") * 0.05)
    w2 = mx.mx_quantize(torch.randn((d, f), generator=g, device="cuda") * 0.05)
    h, packed = mx.residual_norm(x, u, **p, post=True, packed=True)
    hidden = mx.mx_linear_fwd(*packed, *w1, out_dtype=F32)
    out = mx.mx_linear_fwd(*mx.activation(hidden, "silu", gated=True, packed=True), *w2, out_dtype=F32)
    _, y = mx.residual_norm(x.float(), u.float(), **p, post=True)
    y = ref.norm(f64(h), False, EPS, f64(p["pre_weight"]), None)[0]
    deq = lambda q: f64(mx.mx_dequantize(*q))
    want1 = deq(mx.mx_quantize(y.float().cuda())) @ deq(w1).t()
    # a code next to a threshold may differ: such a one moves the product by a step of one of its terms
    assert (f64(hidden) - want1).norm() <= 1e-2 * want1.norm()
    a = ref.act("silu", f64(hidden)[:, :f])[0] * f64(hidden)[:, f:]
    want2 = deq(mx.mx_quantize(a.float().cuda())) @ deq(w2).t()
    assert (f64(out) - want2).norm() <= 1e-2 * want2.norm()


# ---- 8-bit checkpoints ----------------------------------------------------------------------------

@pytest.mark.parametrize("t", [BF, F32])
@pytest.mark.parametrize("n,d", [(1, 1), (3, 5), (7, 31), (64, 32), (9, 33), (197, 192), (50, 1000), (3, 4097), (1030, 96)])
def test_checkpoint_codec(mx, t, n, d):
    g = torch.Generator(device="cuda").manual_seed(n * 1000 + d)
    x = (torch.randn((n, d), generator=g, device="cuda") * torch.exp2(torch.randint(-30, 30, (n, 1), generator=g, device="cuda").float())).to(t)
    codes, scales = mx.mx_checkpoint_pack(x)
    P = (d + 31) // 32 * 32
    assert codes.shape == (n, P) and scales.shape == (n, P // 32)
    want, byte = ref.eight_bits(f64(x))
    assert torch.equal(scales.cpu(), byte)
    assert not codes[:, d:].any()
    back = mx.mx_checkpoint_unpack(codes, scales, d, t)
    assert torch.equal(f64(back), want)
    assert torch.equal(torch.signbit(back), torch.signbit(x))
    other = mx.mx_checkpoint_unpack(codes, scales, d, F32 if t == BF else BF)
    assert torch.equal(f64(other), want)                                    # E4M3 values have four significant bits
    # strided source and destination, given outputs
    wide = torch.full((n, d + 11), 7.0, device="cuda", dtype=t)
    wide[:, 5:5 + d] = x
    out = (torch.full_like(codes, 9), torch.full_like(scales, 9))
    mx.mx_checkpoint_pack(wide[:, 5:5 + d], out=out)
    assert torch.equal(out[0], codes) and torch.equal(out[1], scales)
    wide.fill_(7.0)
    mx.mx_checkpoint_unpack(codes, scales, d, t, out=wide[:, 5:5 + d])
    assert torch.equal(wide[:, 5:5 + d], back) and (wide[:, :5] == 7).all() and (wide[:, 5 + d:] == 7).all()


def test_checkpoint_codec_over_the_whole_domain(mx):
    """Every bf16 value as the largest of its group beside smaller ones, FP32 values on and beside thresholds, zeros."""
    bits = torch.arange(0, 0x7F80, dtype=torch.int32)
    top = (bits << 16).view(torch.float32)
    g = torch.Generator().manual_seed(1)
    x = top[:, None] * torch.rand((len(top), 32), generator=g).mul(2).sub(1)
    x[:, 3], x[:, 4], x[:, 5] = top, -0.0, 0.0
    x = x.to(BF)
    codes, scales = mx.mx_checkpoint_pack(x.cuda())
    want, byte = ref.eight_bits(x)
    # from 31/32 * 2^128 on the nearest E4M3 value is 256 * 2^120 = 2^128, which FP32 has no finite value for
    want = want.float().double()
    assert torch.equal(scales.cpu(), byte) and torch.equal(f64(mx.mx_checkpoint_unpack(codes, scales, 32)), want)
    values = torch.tensor([m / 8 * 2.0 ** -6 for m in range(8)] + [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8)][:-1])
    mids = (values[1:] + values[:-1]) / 2
    near = torch.cat([torch.nextafter(mids, torch.tensor(0.0)), mids, torch.nextafter(mids, torch.tensor(1e9)), values])
    near = torch.cat([near, -near])
    for e in (-100, -20, -1, 0, 3, 60, 110):
        y = torch.zeros((len(near), 32))
        y[:, 0], y[:, 1] = 448.0, near
        y = torch.ldexp(y, torch.tensor(e))
        codes, scales = mx.mx_checkpoint_pack(y.cuda())
        want, byte = ref.eight_bits(y)
        assert torch.equal(scales.cpu(), byte) and torch.equal(f64(mx.mx_checkpoint_unpack(codes, scales, 32)), want), e


def test_checkpoint_of_what_is_not_finite(mx):
    x = torch.ones((3, 64), device="cuda", dtype=BF)
    x[0, 5], x[1, 40], x[2, 1] = float("nan"), float("inf"), float("-inf")
    y = mx.mx_checkpoint_unpack(*mx.mx_checkpoint_pack(x), 64, BF)
    want = torch.ones((3, 64))
    want[0, 5], want[1, 32:], want[2, :32] = float("nan"), float("nan"), float("nan")
    assert torch.equal(torch.isnan(y.cpu()), torch.isnan(want)) and (y.cpu()[~torch.isnan(want)] == 1).all()


# ---- activations ----------------------------------------------------------------------------------

def act_bound(kind, x, err):
    """Error of act(x) and act'(x) that the interface allows."""
    a, s = ref.act(kind, x)
    rel = torch.where(x.abs() <= 4, 2.0 ** -18, 2.0 ** -15)
    return a, s, rel * a.abs().clamp_min(2.0 ** -100)


@pytest.mark.parametrize("kind", ["gelu", "silu"])
@pytest.mark.parametrize("t", [BF, F32])
@pytest.mark.parametrize("ckpt", [False, True])
@pytest.mark.parametrize("gated", [False, True])
def test_activation(mx, kind, t, ckpt, gated):
    for n, f in ((1, 1), (3, 7), (5, 32), (64, 96), (9, 1001), (33, 2048), (2, 8200)):
        print("activation", kind, t, ckpt, gated, n, f, flush=True)
        g = torch.Generator(device="cuda").manual_seed(n + f)
        p = (torch.randn((n, f * (1 + gated)), generator=g, device="cuda") * 2).to(t).requires_grad_(True)
        da = torch.randn((n, f), generator=g, device="cuda").to(t)
        a = mx.activation(p, kind, gated=gated, checkpoint=ckpt)
        with torch.no_grad():
            assert torch.equal(mx.activation(p, kind, gated=gated), a)
        p64, d64 = f64(p), f64(da)
        y, _, err = act_bound(kind, p64[:, :f], None)
        scale = p64[:, f:].abs() if gated else torch.ones_like(y)
        check(a, y * (p64[:, f:] if gated else 1), err * scale / ref.EPS + (y * scale).abs(), 1, "a")
        dp = torch.autograd.grad(a, p, da)[0]
        halves = [p64[:, :f], p64[:, f:]] if gated else [p64]
        if ckpt:
            halves = [ref.eight_bits(q)[0] for q in halves]
        y, s, err = act_bound(kind, halves[0], None)
        # act' is a sum of terms of at most 1 + |x| phi(x) < 1.3 (SiLU 1.2), each within 2^-19
        up = halves[1] if gated else torch.ones_like(y)
        check(dp[:, :f], d64 * up * s, (d64 * up).abs() * 32, 2, "dp")
        if gated:
            check(dp[:, f:], d64 * y, d64.abs() * (err / ref.EPS + y.abs()), 2, "d up")


def test_activation_over_its_domain(mx):
    x = torch.cat([torch.linspace(-20, 20, 400001), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 1e-10, 88.0, -88.0, 100.0, -100.0, 3e18, -3e18, 3e38, -3e38])])
    for kind in ("gelu", "silu"):
        a = mx.activation(x.cuda(), kind).cpu().double()
        want, _, err = act_bound(kind, x.double(), None)
        assert torch.isfinite(a).all()
        tail = 2.0 ** -100                                # exp(-x^2 / 2) and exp(x) reach zero below FP32's range
        assert ((a - want).abs() <= err + 2.0 ** -24 * want.abs() + tail).all(), kind
        p = x.cuda().requires_grad_(True)
        s = torch.autograd.grad(mx.activation(p, kind).sum(), p)[0].cpu().double()
        assert ((s - ref.act(kind, x.double().clamp(-1e4, 1e4))[1]).abs() <= 2.0 ** -18).all(), kind


def test_activation_strides_and_shapes(mx):
    g = torch.Generator(device="cuda").manual_seed(13)
    p = torch.randn((3, 5, 2 * 72), generator=g, device="cuda").to(BF)
    want = mx.activation(p.view(15, 144), "silu", gated=True)
    assert torch.equal(mx.activation(p, "silu", gated=True).view(15, 72), want) and mx.activation(p, "silu", gated=True).shape == (3, 5, 72)
    wide = torch.zeros((15, 150), device="cuda", dtype=BF)
    wide[:, 5:149] = p.view(15, 144)
    assert torch.equal(mx.activation(wide[:, 5:149], "silu", gated=True), want)
    q = wide[:, 5:149].detach().requires_grad_(True)
    for ckpt in (False, True):
        a = mx.activation(q, "silu", gated=True, checkpoint=ckpt)
        got = torch.autograd.grad(a.float().sum(), q)[0]
        r = p.view(15, 144).detach().requires_grad_(True)
        want_g = torch.autograd.grad(mx.activation(r, "silu", gated=True, checkpoint=ckpt), r, torch.ones((15, 72), device="cuda", dtype=BF))[0]
        assert torch.equal(got, want_g)
    assert mx.activation(p[0, 0], "gelu").shape == (144,)


@pytest.mark.parametrize("t,n", [(BF, 9001), (F32, 4501)])
@pytest.mark.parametrize("gated", [False, True])
def test_activation_gradient_beyond_the_cache(mx, t, n, gated):
    """A gradient of 295 MB is that of its rows one by one."""
    g = torch.Generator(device="cuda").manual_seed(12)
    p = torch.randn((n, 16384), generator=g, device="cuda").to(t)
    da = torch.randn((n, 16384 // (1 + gated)), generator=g, device="cuda").to(t)
    for ckpt in (False, True):
        f = lambda p, da: torch.autograd.grad(mx.activation(p.requires_grad_(True), "silu", gated=gated, checkpoint=ckpt), p, da)[0]
        whole = f(p, da)
        for rows in (slice(0, 64), slice(n // 2, n // 2 + 33), slice(n - 65, n)):
            assert torch.equal(whole[rows], f(p[rows].detach().clone(), da[rows].contiguous()))


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("floor", [False, True])
def test_activation_packed(mx, gated, floor):
    mode = mx.SCALE_FLOOR if floor else mx.SCALE_TRUNCFREE
    g = torch.Generator(device="cuda").manual_seed(14)
    for n, f in ((1, 32), (7, 96), (300, 1056)):
        p = torch.randn((n, f * (1 + gated)), generator=g, device="cuda") * 2
        for kind in ("gelu", "silu"):
            codes, scales = mx.activation(p, kind, gated=gated, packed=True, scale_mode=mode)
            want = mx.mx_quantize(mx.activation(p, kind, gated=gated), scale_mode=mode)
            assert torch.equal(codes, want[0]) and torch.equal(scales, want[1])
            bf = mx.activation(p.to(BF), kind, gated=gated, packed=True, scale_mode=mode)
            want = mx.mx_quantize(mx.activation(p.to(BF).float(), kind, gated=gated), scale_mode=mode)
            assert torch.equal(bf[0], want[0]) and torch.equal(bf[1], want[1])


# ---- as they are used -----------------------------------------------------------------------------

def make_block(mx, d, f, gated, checkpoint, dtype=F32):
    lin1 = mx.MxLinear(d, f * (1 + gated), dtype=dtype, flow="microscaling", layer_id=1)
    lin2 = mx.MxLinear(f, d, dtype=dtype, flow="microscaling", layer_id=2)
    norm = mx.MxResidualNorm(d, post=True, gate=0.7, residual_scale=1.1, checkpoint=checkpoint, dtype=dtype)
    act = mx.MxActivation("silu" if gated else "gelu", gated=gated, checkpoint=checkpoint)
    first = mx.MxResidualNorm(d, checkpoint=checkpoint, dtype=dtype)
    params = [t for m in (lin1, lin2, norm, first) for t in m.parameters()]

    def run(x):
        x, y = first(x)
        h, z = norm(x, lin2(act(lin1(y))))
        return h, z
    return run, params


@pytest.mark.parametrize("gated", [False, True])
def test_block_trains_through_the_linear_layers(mx, gated):
    """MLP block: norm, MxLinear, activation, MxLinear, gated residual with norms.  The run of modules gives what the
    operators give one by one, every parameter gets a gradient, and 8-bit checkpoints change the gradients by little."""
    torch.manual_seed(15)
    d, f, n = 96, 128, 200
    run, params = make_block(mx, d, f, gated, False)
    x = torch.randn((n, d), device="cuda").to(BF).requires_grad_(True)
    dh, dz = torch.randn((n, d), device="cuda").to(BF), torch.randn((n, d), device="cuda").to(BF)

    def grads(run):
        h, z = run(x)
        return (h.detach(), z.detach()), torch.autograd.grad((h, z), [x] + params, (dh, dz))
    out, exact = grads(run)
    run8, params8 = make_block(mx, d, f, gated, True)
    with torch.no_grad():
        for a, b in zip(params8, params):
            a.copy_(b)
    params[:] = params8
    out8, eight = grads(run8)
    assert all(torch.equal(a, b) for a, b in zip(out, out8))
    for a, b in zip(exact, eight):
        assert torch.isfinite(b).all() and b.abs().sum() > 0
        # kept values are off by 2^-4 at most and 2^-5.5 in the root of the mean square; the quantizers of the backward
        # pass behind them turn small differences into steps of a quarter of a value
        assert (a.double() - b.double()).norm() <= 0.25 * a.double().norm()


def test_recorded_into_a_graph(mx):
    """Forward and backward captured; each replay, with eager work and synchronizations between, equals the eager result."""
    torch.manual_seed(16)
    n, d, f = 300, 160, 96
    p = {k: torch.randn(d, device="cuda").requires_grad_(True) for k in ("pre_weight", "post_weight", "pre_bias", "post_bias", "gate")}
    xs, us, ps = (torch.randn((n, w), device="cuda").to(BF).requires_grad_(True) for w in (d, d, 2 * f))
    dh, dy, da = (torch.randn((n, w), device="cuda").to(BF) for w in (d, d, f))

    def step():
        h, y = mx.residual_norm(xs, us, **p, norm="layer", post=True, checkpoint=True)
        a = mx.activation(ps, "silu", gated=True, checkpoint=True)
        codes = mx.mx_checkpoint_pack(h.detach())
        with torch.no_grad():
            packed = mx.residual_norm(xs, us, **p, norm="layer", post=True, packed=True)
        return (h, y, a, *torch.autograd.grad((h, y), (xs, us, *p.values()), (dh, dy)), torch.autograd.grad(a, ps, da)[0],
                mx.mx_checkpoint_unpack(*codes, d), *packed[1])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = step()
    for k in range(4):
        with torch.no_grad():
            for t in (xs, us, ps, *p.values()):
                t.copy_(torch.randn_like(t))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.detach().clone() for t in recorded]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k


@pytest.mark.parametrize("d", [8192, 8200, 16384])
def test_wide_rows_recorded_into_a_graph(mx, d):
    torch.manual_seed(19)
    x, u = (torch.randn((600, d), device="cuda").to(BF).requires_grad_(True) for _ in range(2))
    w, v = (torch.randn(d, device="cuda").to(BF).requires_grad_(True) for _ in range(2))
    gate = torch.randn((3, d), device="cuda").to(BF).requires_grad_(True)
    dh, dy = (torch.randn((600, d), device="cuda").to(BF) for _ in range(2))

    def step():
        h, y = mx.residual_norm(x, u, pre_weight=w, post=True, post_weight=v, gate=gate, checkpoint=True)
        return (h, y, *torch.autograd.grad((h, y), (x, u, w, v, gate), (dh, dy)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = step()
    for k in range(3):
        with torch.no_grad():
            for t in (x, u, w, v, gate):
                t.copy_(torch.randn_like(t))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.detach().clone() for t in recorded]
        assert all(torch.equal(a, b) for a, b in zip(got, step())), k


@pytest.mark.parametrize("d", [64, 8200])
def test_c_interface_without_a_block_reads_no_scales(mx, d):
    """u NULL: the norm of x alone, whatever stands in the scales; and its gradient."""
    import ctypes
    B = mx.binding
    x, y, dy, dx = (torch.randn((5, d), device="cuda") for _ in range(4))
    stats, w = torch.zeros((5, 4), device="cuda"), torch.randn(d, device="cuda")
    need = B.lib().mx_residual_norm_workspace_bytes(5, d, 0)
    work = torch.empty(need, device="cuda", dtype=torch.uint8)
    results = []
    for scale in (1.0, 0.0, float("nan")):
        a = B.ResidualNormArgs(rows=5, cols=d, x=x.data_ptr(), y=y.data_ptr(), ldx=d, ldy=d, pre=1, pre_weight=w.data_ptr(), eps=1e-6,
                               residual_scale=scale, branch_scale=scale, stats=stats.data_ptr())
        st = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
        assert B.lib().mx_residual_norm_fwd(ctypes.byref(a), st) == 0
        b = B.ResidualNormGrads(branch=0, dy=dy.data_ptr(), dx=dx.data_ptr(), lddy=d, lddx=d, workspace=work.data_ptr(), workspace_bytes=need)
        assert B.lib().mx_residual_norm_bwd(ctypes.byref(a), ctypes.byref(b), st) == 0
        results.append((y.clone(), dx.clone()))
    leaf = x.clone().requires_grad_(True)
    want = mx.residual_norm(leaf, pre_weight=w)[1]
    (dwant,) = torch.autograd.grad(want, leaf, dy)
    for got in results:
        assert torch.equal(got[0], want.detach()) and torch.equal(got[1], dwant)


def test_two_graphs_and_a_side_stream(mx):
    """Calls on two streams at once and two recorded passes replayed together share no scratch memory."""
    torch.manual_seed(17)
    n, d = 2000, 320
    sets = []
    for _ in range(2):
        x, u = (torch.randn((n, d), device="cuda").to(BF).requires_grad_(True) for _ in range(2))
        w = torch.randn(d, device="cuda").requires_grad_(True)
        sets.append((x, u, w, torch.randn((n, d), device="cuda").to(BF)))

    def step(x, u, w, dy):
        h, y = mx.residual_norm(x, u, pre_weight=w, checkpoint=True)
        return torch.autograd.grad(y, (x, u, w), dy)
    want = [step(*s) for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = []
    for st, s in zip(streams, sets):
        with torch.cuda.stream(st):
            got.append([step(*s) for _ in range(5)])
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(x, y) for r in a for x, y in zip(r, b))
    graphs, outs = [], []
    for s in sets:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step(*s))
        graphs.append(graph)
    for _ in range(3):
        for st, graph in zip(streams, graphs):
            with torch.cuda.stream(st):
                graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_captured_backward_beside_an_eager_graph_of_the_same_leaves(mx):
    """Recording a call on leaves of an eager graph that lives is refused (its backward pass would end the process); with
    that graph gone, or on detached inputs, it is recorded."""
    torch.manual_seed(18)
    x, u = (torch.randn((64, 96), device="cuda").to(BF).requires_grad_(True) for _ in range(2))
    w = torch.randn(96, device="cuda").requires_grad_(True)
    dy = torch.randn((64, 96), device="cuda").to(BF)
    h, y = mx.residual_norm(x, u, pre_weight=w)                            # lives on
    a = mx.activation(u)
    want = torch.autograd.grad(y, (x, u, w), dy, retain_graph=True)
    refusals = []
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for call in (lambda: mx.residual_norm(x, u, pre_weight=w), lambda: mx.activation(u), lambda: mx.activation(a)):
            try:
                call()
            except RuntimeError as e:
                refusals.append(str(e))
        leaves = [t.detach().requires_grad_(True) for t in (x, u, w)]
        h2, y2 = mx.residual_norm(*leaves[:2], pre_weight=leaves[2])
        inside = torch.autograd.grad(y2, leaves, dy)
    assert len(refusals) == 3 and all("another stream" in r for r in refusals)
    del h, y, a
    graph2 = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph2):
        h3, y3 = mx.residual_norm(x, u, pre_weight=w)
        inside2 = torch.autograd.grad(y3, (x, u, w), dy)
    for _ in range(3):
        graph.replay()
        graph2.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) and torch.equal(p, r) for p, q, r in zip(want, inside, inside2))


def test_refusals_that_need_the_device(mx):
    x = torch.ones((4, 64), device="cuda", requires_grad=True)
    with pytest.raises(ValueError):
        mx.residual_norm(x, x, packed=True)
    with pytest.raises(ValueError):
        mx.activation(x, packed=True)
    with pytest.raises(RuntimeError):
        mx.residual_norm(x, torch.ones(4, 64))
    with pytest.raises(RuntimeError):
        mx.residual_norm(x, x, gate=torch.ones(64))
    for call in (lambda: mx.residual_norm(x, x)[1], lambda: mx.activation(x)):
        with pytest.raises(NotImplementedError):
            torch.autograd.grad(call().sum(), x, create_graph=True)
    with pytest.raises(NotImplementedError):
        torch.jit.trace(lambda t: mx.activation(t), (x,))
    # what was kept may not change under the backward pass
    h, y = mx.residual_norm(x, x.detach().clone(), checkpoint=False)
    with torch.no_grad():
        h.add_(1)
    with pytest.raises(RuntimeError, match="modified"):
        y.sum().backward()
    # saved-tensor hooks that hand back something else
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: t[:1]):
        a = mx.activation(x, checkpoint=True)
    with pytest.raises(mx.MxError):
        a.sum().backward()


def test_modules_keep_their_state(mx):
    m = mx.MxResidualNorm(64, norm="layer", post=True, gate=0.3)
    assert set(m.state_dict()) == {"pre_weight", "pre_bias", "post_weight", "post_bias", "gate"}
    m2 = mx.MxResidualNorm(64, norm="layer", post=True, gate=0.1)
    m2.load_state_dict(m.state_dict())
    x = torch.randn((5, 64), device="cuda")
    assert all(torch.equal(a, b) for a, b in zip(m(x, x), m2(x, x)))
    assert set(mx.MxResidualNorm(64).state_dict()) == {"pre_weight"}
    assert set(mx.MxResidualNorm(64, affine=False, post=True).state_dict()) == set()


@pytest.mark.parametrize("d", [40, 41, 1001])
def test_rows_far_apart(mx, d):
    """Rows 2^31 bytes apart, as columns of a large matrix: the results are those of dense rows."""
    g = torch.Generator(device="cuda").manual_seed(21)
    n, ld = 12, (1 << 30) + 3
    far = torch.empty(n * ld, device="cuda", dtype=BF).as_strided((n, d), (ld, 1))
    x, u, p = make(g, n, d, BF, BF, F32, False, True, 3)
    dh, dy = (torch.randn((n, d), generator=g, device="cuda").to(BF) for _ in range(2))

    def step(x, u, dy):
        leaves = [t.detach().requires_grad_(True) for t in (x, u, *p.values())]
        h, y = mx.residual_norm(leaves[0], leaves[1], **dict(zip(p, leaves[2:])), post=True)
        return (h, y, *torch.autograd.grad((h, y), leaves, (dh, dy)))
    want = step(x, u, dy)
    for which in range(3):
        data = [x, u, dy]
        far.copy_(data[which])
        data[which] = far
        assert data[which].stride(0) == ld
        # sums over rows go by another split; the rows themselves do not
        for i, (a, b) in enumerate(zip(step(*data), want)):
            if i < 4:
                assert torch.equal(a, b), (which, i)
            else:
                torch.testing.assert_close(a, b, rtol=2.0 ** -16, atol=2.0 ** -16 * b.abs().max().item())


@pytest.mark.parametrize("off,ld", [(1, 96), (0, 97), (3, 98), (2, 100), (1, 131)])
@pytest.mark.parametrize("t", [BF, F32])
def test_rows_at_any_alignment(mx, t, off, ld):
    """Whole vectors at addresses of no more than their elements' alignment; what lies between the rows stays as it is."""
    g = torch.Generator(device="cuda").manual_seed(22)
    n, d = 70, 96
    x, u, p = make(g, n, d, t, t, F32, True, True, 1)
    place = lambda: torch.full((n * ld + 8,), 7.0, device="cuda", dtype=t)
    mem = {k: place() for k in ("x", "u", "dy")}
    at = {k: m.as_strided((n, d), (ld, 1), off) for k, m in mem.items()}
    dy = torch.randn((n, d), generator=g, device="cuda").to(t)
    for k, v in (("x", x), ("u", u), ("dy", dy)):
        at[k].copy_(v)

    def step(x, u, dy):
        x, u = x.detach().requires_grad_(True), u.detach().requires_grad_(True)
        h, y = mx.residual_norm(x, u, **p, norm="layer", post=True)
        return (h, y, *torch.autograd.grad(y, (x, u), dy))
    assert all(torch.equal(a, b) for a, b in zip(step(at["x"], at["u"], at["dy"]), step(x, u, dy)))
    # outputs there, through the C interface
    import ctypes
    B = mx.binding
    out = {k: place() for k in ("h", "y")}
    want = mx.residual_norm(x, u, post=True)
    bf = int(t == BF)
    a = B.ResidualNormArgs(rows=n, cols=d, x=at["x"].data_ptr(), u=at["u"].data_ptr(), ldx=ld, ldu=ld, ldh=ld, ldy=ld, x_dtype=bf, u_dtype=bf, pre=1, post=1,
                           residual_scale=1.0, branch_scale=1.0, eps=1e-6, **{k: m.data_ptr() + off * t.itemsize for k, m in out.items()})
    assert B.lib().mx_residual_norm_fwd(ctypes.byref(a), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
    for m, w in zip(out.values(), want):
        expected = place()
        expected.as_strided((n, d), (ld, 1), off).copy_(w)
        assert torch.equal(m, expected)


@pytest.mark.parametrize("t", [BF, F32])
@pytest.mark.parametrize("d", [5, 33, 1001, 4099, 9001, 16383])
@pytest.mark.parametrize("post", [False, True])
def test_odd_rows_in_place_and_apart(mx, t, d, post):
    """h over x, and outputs in rows further apart than they are long: only the rows change."""
    import ctypes
    B = mx.binding
    g = torch.Generator(device="cuda").manual_seed(23)
    n, ld = 600, d + 3
    x, u, p = make(g, n, d, t, t, F32, False, post, 1)
    want = mx.residual_norm(x, u, **p, post=post)
    mem = [torch.full((n * ld,), 7.0, device="cuda", dtype=t) for _ in range(2)]
    rows = [m.as_strided((n, d), (ld, 1)) for m in mem]
    rows[0].copy_(x)
    bf = int(t == BF)
    a = B.ResidualNormArgs(rows=n, cols=d, x=mem[0].data_ptr(), h=mem[0].data_ptr(), y=mem[1].data_ptr(), u=u.data_ptr(), ldx=ld, ldu=d, ldh=ld, ldy=ld,
                           x_dtype=bf, u_dtype=bf, pre=1, post=int(post), residual_scale=1.0, branch_scale=1.0, eps=1e-6, gate_rows=1, ld_gate=d,
                           **{k: v.data_ptr() for k, v in p.items()})
    assert B.lib().mx_residual_norm_fwd(ctypes.byref(a), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
    for m, w in zip(mem, want):
        expected = torch.full((n * ld,), 7.0, device="cuda", dtype=t)
        expected.as_strided((n, d), (ld, 1)).copy_(w)
        assert torch.equal(m, expected)


def test_large_offsets(mx):
    """Rows beyond 2^31 elements and 2^32 bytes: the last rows equal those of a small call."""
    n, d = (1 << 31) // 8192 + 40, 8192
    x = torch.empty((n, d), device="cuda", dtype=BF).normal_(generator=torch.Generator(device="cuda").manual_seed(19))
    w = torch.linspace(0.5, 1.5, d, device="cuda")
    with torch.no_grad():
        _, y = mx.residual_norm(x, pre_weight=w)
        _, tail = mx.residual_norm(x[-50:], pre_weight=w)
        assert torch.equal(y[-50:], tail)
        del y
        a = mx.activation(x, "silu", gated=True)
        assert torch.equal(a[-50:], mx.activation(x[-50:], "silu", gated=True))
        del a
        codes, scales = mx.mx_checkpoint_pack(x)
        small = mx.mx_checkpoint_pack(x[-50:])
        assert torch.equal(codes[-50:], small[0]) and torch.equal(scales[-50:], small[1])
        back = mx.mx_checkpoint_unpack(codes, scales, d, BF)
        assert torch.equal(back[-50:], mx.mx_checkpoint_unpack(*small, d, BF))
    del back, codes, scales
    q = x.requires_grad_(True)
    _, y = mx.residual_norm(q, pre_weight=w, checkpoint=True)
    dx = torch.autograd.grad(y, q, x.detach())[0]
    r = x.detach()[-50:].clone().requires_grad_(True)
    _, y2 = mx.residual_norm(r, pre_weight=w, checkpoint=True)
    assert torch.equal(dx[-50:], torch.autograd.grad(y2, r, x.detach()[-50:])[0])
