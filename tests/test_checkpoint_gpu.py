"""Activations in 8 bits: codes and steps bit for bit against the definition, and
the dense transform's gradients from them against 64 bits."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def pyg():
    import paper_1903_02428_amd as m
    assert torch.cuda.is_available()
    m.library()
    return m


def codes_of(x):
    """The definition in numpy: the step by trying exponents upwards, exactly."""
    N, F = x.shape
    nb = -(-F // 32)
    y = np.zeros((N, nb * 32))
    y[:, :F] = x.astype(np.float64)
    y = y.reshape(N, nb, 32)
    with np.errstate(invalid="ignore", over="ignore"):
        top = np.abs(y).max(2)
        bad = ~np.isfinite(y).all(2)
        e = np.full(top.shape, -126)
        for k in range(-125, 123):
            e = np.where(top >= 127.5 * 2.0 ** (k - 1), k, e)
        q = np.rint(np.where(bad[..., None], 0, y) / 2.0 ** e[..., None])
    return q.reshape(N, nb * 32).astype(np.int8), np.where(bad, 255, e + 127).astype(np.uint8)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,F", [(1, 1), (3, 32), (17, 33), (100, 100), (5, 1433), (1000, 64), (2, 7)])
def test_codes_and_restore(pyg, N, F, dtype):
    g = torch.Generator().manual_seed(N * 100 + F)
    x = (torch.randn(N, F, generator=g) * torch.exp(3 * torch.randn(N, 1, generator=g))).to(DT[dtype])
    flat = x.view(-1)
    # borders of the step, zeros, the smallest and largest magnitudes
    special = [0.0, -0.0, 127.5, -127.5, 127.4, 255.0, 2.0 ** -126, 2.0 ** -149, 3.0e38, -1e-38, 0.5, 1.5, 2.5]
    n = min(len(special), flat.numel() // 3)
    flat[:n] = torch.tensor(special[:n]).to(x.dtype)
    if N > 10:
        x[-1, -1], x[-2, 0], x[-3, F // 2] = float("nan"), float("inf"), -float("inf")
        x[-4] = 0.0
    kept = pyg.activation_checkpoint(x.cuda())
    q, e = codes_of(x.float().numpy())
    assert np.array_equal(kept.steps.cpu().numpy(), e) and np.array_equal(kept.codes.cpu().numpy(), q)
    val = q.astype(np.float64).reshape(N, -1, 32) * 2.0 ** (e.astype(np.float64)[..., None] - 127)
    val = np.where(e[..., None] == 255, np.nan, val).reshape(N, -1)[:, :F]
    for out in ("f32", "bf16"):  # exact in both
        got = pyg.checkpoint_restore(kept, DT[out]).float().cpu().numpy()
        assert np.array_equal(got.astype(np.float64), val.astype(np.float32).astype(np.float64), equal_nan=True)
    ok = np.isfinite(val)
    step = 2.0 ** (np.repeat(e, 32, 1)[:, :F].astype(np.float64) - 127)
    assert (np.abs(val - x.double().numpy())[ok] <= step[ok] / 2).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,Fi,Fo", [(1, 1, 1), (31, 16, 7), (300, 33, 64), (1000, 128, 128), (700, 500, 40),
                                     (2111, 130, 257), (50, 1024, 128), (5000, 64, 16)])
def test_dense_backward(pyg, N, Fi, Fo, dtype):
    dt = DT[dtype]
    g = torch.Generator().manual_seed(N + Fi)
    x, go = torch.randn(N, Fi, generator=g).to(dt), torch.randn(N, Fo, generator=g).to(dt)
    theta = torch.randn(Fi, Fo, generator=g).to(dt)
    kept = pyg.activation_checkpoint(x.cuda())
    gx, gt = pyg.dense_transform_backward(go.cuda(), theta.cuda(), kept)
    xr = pyg.checkpoint_restore(kept, torch.float32).cpu().double()
    half = torch.finfo(dt).eps / 2
    for name, got, val, mag, terms in (("grad_theta", gt, xr.T @ go.double(), xr.abs().T @ go.double().abs(), N),
                                       ("grad_x", gx, go.double() @ theta.double().T, go.double().abs() @ theta.double().abs().T, Fo)):
        # products in 32 bits or exact, sums of `terms` (three parts a term) in any order
        bound = (3 * terms + 8) * U * mag
        bound = bound + half * (val.abs() + bound) + 1e-30
        err = (got.cpu().double() - val).abs()
        assert (err <= bound).all(), f"{name}: worst error over bound {float((err / bound).max()):.3g}"
    again = pyg.dense_transform_backward(go.cuda(), theta.cuda(), kept)
    assert torch.equal(gx, again[0]) and torch.equal(gt, again[1])
    only = pyg.dense_transform_backward(go.cuda(), theta.cuda(), kept, need_grad_x=False)
    assert only[0] is None and torch.equal(only[1], gt)


def test_all_bits_of_fp32_gradients(pyg):
    """A gradient's three parts hold it whole: products by one code come back exactly."""
    N, F = 64, 32
    x = torch.zeros(N, F)
    x[5] = 1.0
    go = torch.randn(N, 40, generator=torch.Generator().manual_seed(0)) * torch.logspace(-20, 20, 40)
    go[5, 0], go[5, 1] = 3.4e38, float("inf")
    kept = pyg.activation_checkpoint(x.cuda())
    _, gt = pyg.dense_transform_backward(go.cuda(), torch.zeros(F, 40, device="cuda"), kept)
    assert torch.equal(gt.cpu(), go[5].expand(F, 40))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dense_transform_function(pyg, dtype):
    dt = DT[dtype]
    g = torch.Generator().manual_seed(3)
    x, theta, go = (torch.randn(*s, generator=g).to(dt).cuda() for s in ((200, 48), (48, 80), (200, 80)))
    xl, tl = x.clone().requires_grad_(True), theta.clone().requires_grad_(True)
    out = pyg.DenseTransform.apply(xl, tl)
    assert torch.equal(out, pyg.dense_transform(x, theta, dt))
    gx, gt = torch.autograd.grad(out, [xl, tl], go)
    want = pyg.dense_transform_backward(go, theta, pyg.activation_checkpoint(x))
    assert torch.equal(gx, want[0]) and torch.equal(gt, want[1])
    kept = pyg.activation_checkpoint(x)
    out = pyg.DenseTransform.apply(xl, tl, kept)
    assert torch.equal(torch.autograd.grad(out, [tl], go)[0], gt)
    out = pyg.DenseTransform.apply(xl, theta)
    assert torch.equal(torch.autograd.grad(out, [xl], go)[0], gx)
    with pytest.raises(ValueError):
        pyg.DenseTransform.apply(xl, tl, pyg.activation_checkpoint(x[:100].contiguous()))


def test_empty_and_refusals(pyg):
    z = torch.zeros(0, 40, device="cuda")
    kept = pyg.activation_checkpoint(z)
    assert pyg.checkpoint_restore(kept).shape == (0, 40)
    gx, gt = pyg.dense_transform_backward(torch.zeros(0, 5, device="cuda"), torch.ones(40, 5, device="cuda"), kept)
    assert gx.shape == (0, 40) and (gt == 0).all()
    x = torch.randn(8, 40, device="cuda")
    for bad in (x.half(), x.t(), x.cpu(), x[0]):
        with pytest.raises(ValueError):
            pyg.activation_checkpoint(bad)
    kept = pyg.activation_checkpoint(x)
    with pytest.raises(ValueError):
        pyg.activation_checkpoint(x[:4].contiguous(), out=kept)
    g, t = torch.zeros(8, 5, device="cuda"), torch.zeros(40, 5, device="cuda")
    for args in ((g, t[:39].contiguous(), kept), (g[:4], t, kept), (g.bfloat16(), t, kept), (g, t, pyg.Checkpoint(kept.codes, kept.steps, 70, torch.float32)),
                 (g, t, pyg.Checkpoint(kept.codes[:, :32].contiguous(), kept.steps, 40, torch.float32))):
        with pytest.raises(ValueError):
            pyg.dense_transform_backward(*args)
    with pytest.raises(ValueError):
        pyg.checkpoint_restore(kept, torch.float16)


def test_written_again_is_noticed(pyg):
    """Arrays that autograd holds and a call writes again: the backward says so and does not use the new values."""
    x = torch.randn(40, 64, device="cuda")
    theta = torch.randn(64, 8, device="cuda", requires_grad=True)
    kept = pyg.activation_checkpoint(x)
    out = pyg.DenseTransform.apply(x, theta, kept)
    pyg.activation_checkpoint(2 * x, out=kept)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(out, [theta], torch.ones_like(out))
    out = pyg.DenseTransform.apply(x, theta, kept)  # and of what is there now it is right
    want = pyg.dense_transform_backward(torch.ones_like(out), theta.detach(), kept, need_grad_x=False)[1]
    assert torch.equal(torch.autograd.grad(out, [theta], torch.ones_like(out))[0], want)
    saved = torch.randn(40, 64, device="cuda", requires_grad=True).exp()
    pyg.checkpoint_restore(kept, out=saved.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(saved, [saved.grad_fn.next_functions[0][0].variable], torch.ones_like(saved))
    saved = torch.randn(5, 2, 8, device="cuda", requires_grad=True).exp()
    qkv = torch.randn(5, 2, 8, device="cuda")
    pyg.global_attention(qkv, qkv, qkv, torch.tensor([0, 5], device="cuda"), out=saved.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(saved, [saved.grad_fn.next_functions[0][0].variable], torch.ones_like(saved))
    with torch.inference_mode():  # arrays without versions are written as they are
        kept = pyg.activation_checkpoint(x)
        pyg.activation_checkpoint(x, out=kept)
        pyg.checkpoint_restore(kept, out=torch.empty_like(x))


def test_input_gradient_of_single_products(pyg):
    """fp32 grad_x of one term a value is the product itself to within the matrix cores' last addition: operands as
    three bf16 parts each, the part products that are left out below 2^-24 of the whole (half a step
    of fp32), the six that are taken exact, summed from the smallest on: one step (two half steps,
    should the sum be cut and not rounded) for the last addition, at most half of one half step for those before."""
    g = torch.Generator().manual_seed(9)
    bits = (torch.randint(0, 1 << 23, (1500 + 300,), generator=g, dtype=torch.int32) | 0x3F800000)
    bits[:8] = bits[1500:1508] = torch.tensor([0x3F80FFFF, 0x3F808000, 0x3F807FFF, 0x3F800001, 0x3FFFFFFF, 0x3FFF7FFF, 0x3F8080FF, 0x3F800000],
                                              dtype=torch.int32)
    val = bits.view(torch.float32)
    sign = torch.where(torch.rand(len(val), generator=g) < 0.5, -1.0, 1.0)
    go, theta = (val * sign)[:1500, None].contiguous(), (val * sign)[1500:, None].contiguous()
    gx, _ = pyg.dense_transform_backward(go.cuda(), theta.cuda(), None, need_grad_theta=False)
    want = go.double() @ theta.double().T
    err = (gx.cpu().double() - want).abs() / want.abs()
    assert float(err.max()) <= 3.5 * U, f"{float(err.max() / U):.2f} half steps"


def test_parts_of_extreme_values(pyg):
    """Cutting fp32 operands into parts keeps the largest values finite, and NaN whatever its bits."""
    top = torch.finfo(torch.float32).max
    go = torch.tensor([top, -top, 3.4e38, 1.0, 0.0, 2.0 ** -90])[:, None]
    theta = torch.ones(4, 1)
    gx, _ = pyg.dense_transform_backward(go.cuda(), theta.cuda(), None, need_grad_theta=False)
    assert torch.equal(gx.cpu(), go.expand(6, 4))
    nan = torch.tensor([0x7F800001, -0x007FFFFF, 0x7FC00000], dtype=torch.int32).view(torch.float32)[:, None].contiguous()
    assert torch.isnan(nan).all()
    gx, _ = pyg.dense_transform_backward(nan.cuda(), theta.cuda(), None, need_grad_theta=False)
    assert torch.isnan(gx).all()
    x = torch.ones(3, 32)
    _, gt = pyg.dense_transform_backward(torch.cat([nan[:1], torch.ones(2, 1)]).cuda(), torch.ones(32, 1, device="cuda"),
                                         pyg.activation_checkpoint(x.cuda()))
    assert torch.isnan(gt).all()


def test_largest_error_of_a_block(pyg):
    """Half a step is up to 1 / 127.5 of a block's largest magnitude: 127.5 takes steps of 2, and 1 comes back as 0."""
    x = torch.full((2, 32), 1.0)
    x[0, 0], x[1, 0] = 127.5, 127.4375
    got = pyg.checkpoint_restore(pyg.activation_checkpoint(x.cuda())).cpu()
    assert (got[0, 1:] == 0).all() and got[0, 0] == 128 and torch.equal(got[1], torch.tensor([127.0] + [1.0] * 31))
