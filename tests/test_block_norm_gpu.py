"""The norms around a block with its gate and residual scale, forward and
gradients, against the formulas in 64 bits, value by value: every width class
(16 lanes a row to a workgroup), odd widths, parts left out, both norms and types."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
NAMES = ("h", "residual", "gate", "scale", "post_weight", "post_bias", "weight", "bias")
U = 2.0 ** -24


@pytest.fixture(scope="module")
def pyg():
    import paper_1903_02428_amd as m
    assert torch.cuda.is_available()
    m.library()
    return m


def make(seed, N, F, dtype, gate, parts, offset=0.0):
    g = torch.Generator().manual_seed(seed)
    t = {"h": torch.randn(N, F, generator=g) + offset, "residual": 2 * torch.randn(N, F, generator=g),
         "gate": torch.randn(N, 1 if gate == "row" else F, generator=g)}
    t = {n: v.to(dtype) for n, v in t.items()}
    for n in NAMES[3:]:
        t[n] = torch.randn(F, generator=g)
    if gate == "none":
        t["gate"] = None
    for n in NAMES:
        if n not in parts and n not in ("h", "gate"):
            t[n] = None
    return t, torch.randn(N, F, generator=g).to(dtype), torch.randn(N, F, generator=g).to(dtype)


def reference(t, gr, gy, layer, eps):
    """{name: (value, bound)}. Every fp32 sum of a row of F terms is off by at most F + 32 half
    steps of the sum of magnitudes (the further operations on a value among the 32), a
    normalised value by that of itself plus one, times what subtracting the mean amplifies."""
    F, N = t["h"].shape[1], t["h"].shape[0]
    d = {n: None if v is None else v.double() for n, v in t.items()}
    half = torch.finfo(t["h"].dtype).eps / 2

    def normed(x, xmag):
        mean = x.mean(1, keepdim=True) if layer else 0.0
        c = x - mean
        rstd = 1 / (c.square().mean(1, keepdim=True) + eps).sqrt()
        n = c * rstd
        return n, rstd, n.abs() + (xmag + (xmag.mean(1, keepdim=True) if layer else 0)) * rstd + \
            n.abs() * ((n.abs() + 1) * xmag * rstd).mean(1, keepdim=True)

    def through(v, vm, n, nm, rstd):
        tn, tm = (v * n).mean(1, keepdim=True), v.mean(1, keepdim=True) if layer else 0.0
        m = rstd * (vm + nm * (vm * nm).mean(1, keepdim=True) * 2 + (vm.mean(1, keepdim=True) if layer else 0))
        return (v - n * tn - tm) * rstd, m * (1 + nm.square().mean(1, keepdim=True))
    u, um = d["h"], d["h"].abs()
    if d["post_weight"] is not None:
        nh, rh, nhm = normed(d["h"], d["h"].abs())
        b = 0.0 if d["post_bias"] is None else d["post_bias"]
        u, um = nh * d["post_weight"] + b, nhm * d["post_weight"].abs() + abs(b)
    sg = torch.sigmoid(d["gate"]) if d["gate"] is not None else torch.ones(1, 1, dtype=torch.float64)
    sgm = sg * (1 + (0.0 if d["gate"] is None else d["gate"].abs()))
    sc = d["scale"] if d["scale"] is not None else torch.ones(F, dtype=torch.float64)
    res = d["residual"] if d["residual"] is not None else torch.zeros(1, F, dtype=torch.float64)
    r, rm = res + sc * sg * u, res.abs() + sc.abs() * sgm * um
    z, m = {"r": r}, {"r": rm}
    t_, tm_ = (torch.zeros_like(r), torch.zeros_like(r)) if gr is None else (gr.double(), gr.double().abs())
    if d["weight"] is not None:
        nr, rr, nrm = normed(r, rm)
        b = 0.0 if d["bias"] is None else d["bias"]
        z["y"], m["y"] = nr * d["weight"] + b, nrm * d["weight"].abs() + abs(b)
        if gy is not None:
            g = gy.double()
            z["grad_weight"], m["grad_weight"] = (g * nr).sum(0), (g.abs() * nrm).sum(0)
            z["grad_bias"], m["grad_bias"] = g.sum(0), g.abs().sum(0)
            v, vm = through(g * d["weight"], (g * d["weight"]).abs(), nr, nrm, rr)
            t_, tm_ = t_ + v, tm_ + vm
    z["grad_residual"], m["grad_residual"] = t_, tm_
    z["grad_scale"], m["grad_scale"] = (t_ * sg * u).sum(0), (tm_ * sgm * um).sum(0)
    dg, dgm = t_ * sc * u * sg * (1 - sg), tm_ * sc.abs() * um * sgm
    if d["gate"] is not None and d["gate"].shape[1] == 1:
        dg, dgm = dg.sum(1, keepdim=True), dgm.sum(1, keepdim=True)
    z["grad_gate"], m["grad_gate"] = dg, dgm
    t_, tm_ = t_ * sc * sg, tm_ * sc.abs() * sgm
    if d["post_weight"] is not None:
        z["grad_post_weight"], m["grad_post_weight"] = (t_ * nh).sum(0), (tm_ * nhm).sum(0)
        z["grad_post_bias"], m["grad_post_bias"] = t_.sum(0), tm_.sum(0)
        t_, tm_ = through(t_ * d["post_weight"], tm_ * d["post_weight"].abs(), nh, nhm, rh)
    z["grad_h"], m["grad_h"] = t_, tm_
    out = {}
    for n, v in z.items():
        rows = n in ("r", "y", "grad_h", "grad_residual", "grad_gate")
        bound = (F + 32 + (0 if rows else N)) * U * m[n]
        out[n] = (v, bound + ((half if rows else U) * (v.abs() + bound)) + 1e-30)
    return out


def check(got, ref, what):
    for n, v in got.items():
        val, bound = ref[n]
        err = (v.detach().cpu().double() - val).abs()
        assert err.shape == val.shape and bool((err <= bound).all()), \
            f"{what} {n}: worst error over bound {float((err / bound).max()):.3g}"


ALL = NAMES
CASES = [  # rows, features, norm, gate, parts
    (1, 64, "layer", "full", ALL),
    (37, 16, "rms", "row", ALL),
    (300, 33, "layer", "row", ALL),
    (129, 128, "rms", "full", ("residual", "scale", "post_weight", "weight")),
    (50, 7, "layer", "none", ("residual", "weight")),
    (70, 250, "layer", "full", ("residual", "scale", "weight", "bias")),
    (33, 512, "rms", "none", ("weight",)),
    (20, 1000, "layer", "row", ALL),
    (9, 1433, "layer", "none", ("residual", "scale", "weight", "bias")),
    (5, 2048, "rms", "full", ALL),
    (6, 4097, "layer", "row", ALL),
    (3, 8192, "layer", "full", ALL),
    (40, 1, "rms", "full", ALL),
    (11, 96, "layer", "full", ("residual", "post_weight")),
    (700, 900, "layer", "full", ALL),
    (600, 1600, "rms", "row", ALL),
    (530, 3000, "layer", "full", ("residual", "scale", "weight", "bias")),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_forward_and_gradients(pyg, i, dtype):
    N, F, norm, gate, parts = CASES[i]
    t, gr, gy = make(i, N, F, DT[dtype], gate, parts)
    dev = {n: None if v is None else v.cuda().requires_grad_(True) for n, v in t.items()}
    r, y, kept = pyg.BlockNorm.apply(*[dev[n] for n in NAMES], norm, 1e-5, t["weight"] is not None)
    names = [n for n in NAMES if dev[n] is not None]
    outs, gouts = ([r, y], [gr.cuda(), gy.cuda()]) if y is not None else ([r], [gr.cuda()])
    grads = torch.autograd.grad(outs, [dev[n] for n in names], gouts)
    got = {"r": r, **({"y": y} if y is not None else {}), **{"grad_" + n: g for n, g in zip(names, grads)}}
    check(got, reference(t, gr, gy if y is not None else None, norm == "layer", 1e-5), f"case {i} {dtype}")
    if kept is not None:
        again = pyg.activation_checkpoint(y.detach())
        assert torch.equal(kept.codes, again.codes) and torch.equal(kept.steps, again.steps)
    # one gradient missing
    if y is not None:
        r, y, _ = pyg.BlockNorm.apply(*[dev[n] for n in NAMES], norm, 1e-5)
        grads = torch.autograd.grad(y, [dev[n] for n in names], gy.cuda())
        check({"grad_" + n: g for n, g in zip(names, grads)}, reference(t, None, gy, norm == "layer", 1e-5), "y alone")


def test_many_rows(pyg):
    """More rows than the backward's workgroups hold at once, and rows far from zero."""
    for N, F, offset in ((40_001, 20, 0.0), (5000, 700, 3.0)):
        t, gr, gy = make(N, N, F, torch.float32, "row", ALL, offset)
        dev = {n: None if v is None else v.cuda() for n, v in t.items()}
        r, y, _ = pyg.block_norm(*[dev[n] for n in NAMES])
        grads = pyg.block_norm_backward(gr.cuda(), gy.cuda(), *[dev[n] for n in NAMES])
        check({"r": r, "y": y, **{"grad_" + n: g for n, g in zip(NAMES, grads)}}, reference(t, gr, gy, True, 1e-5), str(N))
        again = pyg.block_norm_backward(gr.cuda(), gy.cuda(), *[dev[n] for n in NAMES])
        assert all(torch.equal(a, b) for a, b in zip(grads, again))


def test_constant_and_masked_rows(pyg):
    """Rows of one value (variance 0), zero rows, gates at both ends."""
    N, F = 6, 48
    t, gr, gy = make(2, N, F, torch.float32, "full", ALL)
    t["h"][0], t["h"][1] = 0.0, 4.0
    t["residual"][2] = 0.0
    t["gate"][3], t["gate"][4] = -200.0, 200.0
    dev = {n: v.cuda() for n, v in t.items()}
    for norm in ("layer", "rms"):
        r, y, _ = pyg.block_norm(*[dev[n] for n in NAMES], norm=norm)
        grads = pyg.block_norm_backward(gr.cuda(), gy.cuda(), *[dev[n] for n in NAMES], norm=norm)
        ref = reference(t, gr, gy, norm == "layer", 1e-5)
        check({"r": r, "y": y, **{"grad_" + n: g for n, g in zip(NAMES, grads)}}, ref, norm)
        # what one row holds does not reach another
        bad = {n: v.clone() for n, v in dev.items()}
        bad["h"][5] = float("nan")
        r2, y2, _ = pyg.block_norm(*[bad[n] for n in NAMES], norm=norm)
        assert torch.equal(r2[:5], r[:5]) and torch.equal(y2[:5], y[:5]) and torch.isnan(y2[5]).all()


def test_gradients_by_differences(pyg):
    t, gr, gy = make(4, 5, 12, torch.float32, "row", ALL)
    dev = {n: v.cuda() for n, v in t.items()}
    grads = pyg.block_norm_backward(gr.cuda(), gy.cuda(), *[dev[n] for n in NAMES])
    rng = np.random.default_rng(0)

    def loss(p):
        r, y, _ = pyg.block_norm(*[p[n] for n in NAMES])
        return float((r.double().cpu() * gr).sum() + (y.double().cpu() * gy).sum())
    for n, g in zip(NAMES, grads):
        step = torch.from_numpy(rng.standard_normal(t[n].shape).astype(np.float32))
        eps = 2.0 ** -8
        num = (loss({**dev, n: dev[n] + eps * step.cuda()}) - loss({**dev, n: dev[n] - eps * step.cuda()})) / (2 * eps)
        ana = float((g.double().cpu() * step).sum())
        assert abs(num - ana) <= 2e-3 * max(1.0, abs(ana)), n


def test_empty_and_plain(pyg):
    w = torch.ones(8, device="cuda")
    z = torch.zeros(0, 8, device="cuda")
    r, y, kept = pyg.block_norm(z, weight=w, checkpoint=True)
    assert r.shape == y.shape == (0, 8) and kept.N == 0
    grads = pyg.block_norm_backward(z, z, z, weight=w)
    assert (grads[6] == 0).all()
    x = torch.randn(3, 8, device="cuda")
    assert pyg.block_norm(x)[0] is x
    leaf = x.clone().requires_grad_(True)
    r, y, _ = pyg.BlockNorm.apply(leaf, None, None, None, None, None, w)
    g, = torch.autograd.grad([r, y], [leaf], [torch.ones_like(x), torch.zeros_like(x)])
    assert torch.equal(g, torch.ones_like(x))


def test_refusals(pyg):
    x, w = torch.randn(4, 8, device="cuda"), torch.ones(8, device="cuda")
    ok = dict(h=x, residual=x, weight=w)
    for change in (dict(h=x.half()), dict(h=x.cpu()), dict(h=x.t()), dict(residual=x[:2]), dict(residual=x.bfloat16()),
                   dict(gate=x[:, :2].contiguous()), dict(gate=x[:2]), dict(scale=w[:4]), dict(scale=w.bfloat16()), dict(bias=w, weight=None),
                   dict(post_bias=w), dict(norm="batch"), dict(eps=-1.0), dict(weight=None, checkpoint=True)):
        with pytest.raises(ValueError):
            pyg.block_norm(**{**ok, **change})
    with pytest.raises(pyg.PygError):
        pyg.block_norm(torch.zeros(1, 8193, device="cuda"), weight=torch.ones(8193, device="cuda"))
    with pytest.raises(ValueError):
        pyg.block_norm_backward(None, None, x, weight=w)
    with pytest.raises(ValueError):
        pyg.block_norm_backward(None, x, x)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [False, True])
def test_gate_gradient_far_from_zero(pyg, rows, dtype):
    """d sigmoid = sigmoid(x) sigmoid(-x) keeps its bits where sigmoid(x) is nearly one. Of all-positive
    terms: the exponent's argument x log2 e is off by two half steps (the constant's and the product's rounding), so
    each of the two factors by 2 |x| half steps at most; exp2, the reciprocal (a whole step each) and
    the sum in each, the other products and a row's sum of F terms are the rest."""
    F = 24
    x = torch.tensor([-80.0, -40, -17, -12, -3, 0, 3, 8, 12, 15, 17, 20, 25, 40, 60, 80])
    g = torch.Generator().manual_seed(5)
    h, gr = (torch.rand(len(x), F, generator=g).to(DT[dtype]) + 0.5 for _ in range(2))
    gate = (x[:, None] if rows else x[:, None].expand(-1, F)).contiguous().to(DT[dtype])
    scale = torch.rand(F, generator=g) + 0.5
    got = pyg.block_norm_backward(gr.cuda(), None, h.cuda(), gate=gate.cuda(), scale=scale.cuda())[2].cpu().double()
    xd = gate.double()
    want = gr.double() * scale.double() * h.double() * torch.sigmoid(xd) * torch.sigmoid(-xd)
    want = want.sum(1, keepdim=True) if rows else want
    half = 0.0 if dtype == "f32" else torch.finfo(torch.bfloat16).eps / 2
    bound = ((4 * xd.abs() + 16 + (F if rows else 0)) * U + half) * want
    assert ((got - want).abs() <= bound).all(), ((got - want).abs() / bound).amax(1)
