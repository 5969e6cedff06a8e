"""Attention over the graphs of a batch with a bias by relative position, forward
and gradients, against the formulas in 64 bits: every kernel (few queries,
small graphs, large ones), types, head layouts, widths, ragged and empty graphs,
strides, masks that leave rows empty."""
import math

import numpy as np
import pytest
import torch

from tests.attention_reference import attention, close

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def pyg():
    import paper_1903_02428_amd as m
    assert torch.cuda.is_available()
    m.library()
    return m


def ptr_of(n):
    return torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int64, device="cuda")


def inputs(seed, qn, kn, H, Hkv, D, dtype, buckets, reach, causal, pyg, extra=0):
    g = torch.Generator().manual_seed(seed)
    q, grad = (torch.randn(sum(qn) + extra, H, D, generator=g).to(dtype) for _ in range(2))
    k, v = (torch.randn(sum(kn) + extra, Hkv, D, generator=g).to(dtype) for _ in range(2))
    table = torch.randn(buckets, H, generator=g).to(dtype) if buckets else None
    lut = pyg.relative_buckets(buckets, reach, not causal, "cpu") if buckets else None
    return q, k, v, grad, table, lut


def run(pyg, q, k, v, grad, table, lut, qn, kn, causal, scale=None, same=False):
    dev = [t.cuda().requires_grad_(True) for t in (q, k, v)]
    tab = table.cuda().requires_grad_(True) if table is not None else None
    ptr = ptr_of(qn)
    out = pyg.GlobalAttention.apply(*dev, tab, ptr, None if same else ptr_of(kn), lut.cuda() if lut is not None else None,
                                    causal, scale)
    leaves = dev + ([tab] if tab is not None else [])
    grads = torch.autograd.grad(out, leaves, grad.cuda())
    names = ["grad_q", "grad_k", "grad_v"] + (["grad_table"] if tab is not None else [])
    torch.cuda.synchronize()
    return {"out": out, **dict(zip(names, grads))}


# queries and keys of every graph, heads, key heads, features, buckets, reach, causal
CASES = [
    # few queries a graph: one each, none, several, grouped heads in one tile and over several
    ([1, 1, 1], [5, 1, 40], 4, 4, 16, 8, 16, False),
    ([1, 0, 1, 2], [300, 7, 0, 2], 4, 1, 64, 8, 16, True),
    ([3, 1, 9], [1000, 33, 64], 8, 2, 128, 32, 128, True),
    ([1], [5000], 16, 2, 128, 32, 128, False),
    ([2], [2049], 1, 1, 24, 0, 0, True),
    ([1, 17], [100, 31], 20, 1, 40, 4, 8, False),
    # more of them over a long history: several tiles of 16 rows, and many heads on one key head
    ([40, 3], [2600, 90], 2, 1, 64, 8, 16, True),
    ([1], [1500], 40, 1, 32, 8, 64, True),
    # small graphs: a wavefront each
    ([25, 1, 32, 33, 0, 18], None, 4, 4, 16, 16, 32, False),
    ([40, 20, 7], None, 8, 8, 8, 8, 16, True),
    ([31, 64, 65], [40, 10, 100], 2, 1, 80, 8, 8, True),
    ([50, 3], [0, 200], 3, 3, 33, 16, 20, False),
    # large graphs: four wavefronts, several tiles, tiles beyond the reach
    ([200, 1, 129], None, 2, 2, 64, 32, 24, False),
    ([300], None, 4, 2, 128, 32, 128, True),
    ([257], [700], 2, 1, 128, 8, 16, True),
    ([700], [257], 2, 2, 32, 8, 16, True),
    ([130, 250], None, 3, 1, 7, 2, 1, False),
    ([190], [333], 1, 1, 1, 0, 0, False),
    # the largest reach and the most buckets, beside the widest heads
    ([140, 20], None, 1, 1, 128, 1024, 1024, False),
    ([30, 20], None, 1, 1, 128, 1024, 1024, True),
    ([1, 2], [40, 1500], 2, 1, 128, 1024, 1024, True),
    # heads of a group dealt out over workgroups (few key tiles): all of them, and a part
    ([150, 140], None, 6, 1, 40, 8, 16, True),
    ([260], [140], 8, 2, 64, 4, 8, False),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_forward_and_gradients(pyg, i, dtype):
    qn, kn, H, Hkv, D, buckets, reach, causal = CASES[i]
    same = kn is None
    kn = qn if same else kn
    q, k, v, grad, table, lut = inputs(i, qn, kn, H, Hkv, D, DT[dtype], buckets, reach, causal, pyg)
    got = run(pyg, q, k, v, grad, table, lut, qn, kn, causal, same=same)
    close(got, attention(q, k, v, qn, kn, table, lut, causal, grad=grad), f"case {i} {dtype}")
    # without gradients: the same kernels, no statistics kept
    out = pyg.global_attention(q.cuda(), k.cuda(), v.cuda(), ptr_of(qn), ptr_of(kn),
                               None if table is None else table.cuda(), None if lut is None else lut.cuda(), causal)
    assert torch.equal(out, got["out"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_packed_views_and_scale(pyg, dtype):
    # q, k, v as views into one product's rows, and k, v with heads outside rows
    n, H, D = [70, 90], 4, 32
    g = torch.Generator().manual_seed(1)
    qkv = torch.randn(sum(n), 3 * H, D, generator=g).to(DT[dtype])
    grad = torch.randn(sum(n), H, D, generator=g).to(DT[dtype])
    q, k, v = qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:]
    ref = attention(q, k, v, n, n, scale=0.3, grad=grad)
    dev = qkv.cuda()
    views = [dev[:, :H], dev[:, H:2 * H], dev[:, 2 * H:]]
    kv = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in views[1:]]
    for x, y, z in (views, [views[0], *kv]):
        leaves = [t.detach().requires_grad_(True) for t in (x, y, z)]
        out = pyg.GlobalAttention.apply(*leaves, None, ptr_of(n), None, None, False, 0.3)
        grads = torch.autograd.grad(out, leaves, grad.cuda())
        close({"out": out, **dict(zip(("grad_q", "grad_k", "grad_v"), grads))}, ref, f"strides {y.stride()}")
    # odd offsets: no 16-byte rows
    wide = torch.zeros(sum(n), 3 * H, D + 1, dtype=DT[dtype], device="cuda")
    wide[:, :, 1:] = dev
    leaves = [wide[:, i * H:(i + 1) * H, 1:].detach().requires_grad_(True) for i in range(3)]
    out = pyg.GlobalAttention.apply(*leaves, None, ptr_of(n), None, None, False, 0.3)
    grads = torch.autograd.grad(out, leaves, grad.cuda())
    close({"out": out, **dict(zip(("grad_q", "grad_k", "grad_v"), grads))}, ref, "odd offsets")


@pytest.mark.parametrize("qn,kn", [([1, 2], [50, 90]), ([20, 45], [50, 90]), ([150, 3], [200, 130])])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("low", [-math.inf, "lowest"])
def test_masking_buckets(pyg, qn, kn, dtype, low):
    """Buckets of -infinity mask (rows whose keys all are give zeros and zero
    gradients); buckets of the type's lowest value leave a row's keys alike."""
    H, D, reach = 2, 32, 4
    dt = DT[dtype]
    low = torch.finfo(dt).min if low == "lowest" else low
    q, k, v, grad, table, lut = inputs(3, qn, kn, H, 2, D, dt, 8, reach, False, pyg)
    table[:, 0] = low          # head 0: nothing but masks
    table[4:, 1] = low         # head 1: later keys are masked
    table[3, 1] = low          # and the farthest earlier ones
    got = run(pyg, q, k, v, grad, table, lut, qn, kn, False)
    ref = attention(q, k, v, qn, kn, table, lut, False, grad=grad)
    for name, t in got.items():
        assert torch.isfinite(t).all(), name
    close(got, ref, f"{low} {dtype}")


def test_rows_of_no_graph(pyg):
    """Rows behind the last graph: zeros in results made here, left alone in a caller's."""
    for qn, kn in (([1, 1], [40, 9]), ([20, 30], [20, 30]), ([200], [200])):
        q, k, v, grad, table, lut = inputs(5, qn, kn, 2, 2, 16, torch.float32, 8, 16, False, pyg, extra=100)
        k[sum(kn):], v[sum(kn):], q[sum(qn):] = math.nan, math.nan, math.nan
        got = run(pyg, q, k, v, grad, table, lut, qn, kn, False)
        ref = attention(q[:sum(qn)], k[:sum(kn)], v[:sum(kn)], qn, kn, table, lut, False, grad=grad[:sum(qn)])
        for name, t in got.items():
            n = len(ref[name][0])
            assert (t[n:] == 0).all(), name
            close({name: t[:n]}, ref, "padded")
        out = torch.full(q.shape, 7.0, device="cuda")
        pyg.global_attention(q.cuda(), k.cuda(), v.cuda(), ptr_of(qn), ptr_of(kn), table.cuda(), lut.cuda(), out=out)
        assert (out[sum(qn):] == 7).all() and torch.equal(out[:sum(qn)], got["out"][:sum(qn)])


def test_no_leak_between_graphs(pyg):
    """NaN and infinities in one graph do not reach another that shares its tiles."""
    for n in ([20, 30, 25], [150, 200, 90]):
        q, k, v, grad, table, lut = inputs(6, n, n, 2, 2, 16, torch.bfloat16, 8, 16, False, pyg)
        clean = run(pyg, q, k, v, grad, table, lut, n, n, False)
        a, b = n[0], n[0] + n[1]
        for t in (q, k, v):
            t[a:b] = math.inf
            t[a + 1] = math.nan
        bad = run(pyg, q, k, v, grad, table, lut, n, n, False)
        for name in ("out", "grad_q", "grad_k", "grad_v"):
            assert torch.equal(bad[name][:a], clean[name][:a]) and torch.equal(bad[name][b:], clean[name][b:]), name
            assert not torch.isfinite(bad[name][a:b]).all()


def test_gradients_by_differences(pyg):
    n, H, D = [6, 9], 2, 8
    q, k, v, grad, table, lut = inputs(8, n, n, H, 1, D, torch.float32, 8, 8, True, pyg)
    got = run(pyg, q, k, v, grad, table, lut, n, n, True)

    def loss(*t):
        o = pyg.global_attention(*[x.cuda() for x in t[:3]], ptr_of(n), None, t[3].cuda(), lut.cuda(), True)
        return float((o.double().cpu() * grad).sum())
    rng = np.random.default_rng(0)
    base = [q, k, v, table]
    for i, name in enumerate(("grad_q", "grad_k", "grad_v", "grad_table")):
        step = torch.from_numpy(rng.standard_normal(base[i].shape).astype(np.float32))
        eps = 2.0 ** -7
        plus, minus = ([t + s * eps * step if j == i else t for j, t in enumerate(base)] for s in (1, -1))
        num = (loss(*plus) - loss(*minus)) / (2 * eps)
        ana = float((got[name].double().cpu() * step).sum())
        # third-order term of the difference, and fp32 outputs over 2 eps
        assert abs(num - ana) <= 2e-3 * max(1.0, abs(ana)), name


def test_repeatable_and_captured(pyg):
    """The same bits every time, also from a captured graph on another stream
    that replays after other work used the caller's workspace."""
    for qn, kn, D in (([1, 1], [3000, 100], 128), ([60, 200, 90], [60, 200, 90], 64)):
        q, k, v, grad, table, lut = inputs(9, qn, kn, 4, 2, D, torch.bfloat16, 32, 64, True, pyg)
        first = run(pyg, q, k, v, grad, table, lut, qn, kn, True)
        for _ in range(3):
            again = run(pyg, q, k, v, grad, table, lut, qn, kn, True)
            assert all(torch.equal(first[n], again[n]) for n in first)
        dev = [t.cuda() for t in (q, k, v)]
        args = (ptr_of(qn), ptr_of(kn), table.cuda(), lut.cuda(), True)
        gd, out = grad.cuda(), torch.zeros(q.shape, dtype=q.dtype, device="cuda")
        stat, rest = torch.zeros((*q.shape[:2], 2), device="cuda"), torch.zeros_like(out)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            pyg.global_attention(*dev, *args, out=out, stat=stat, rest=rest)
            pyg.global_attention_backward(gd, *dev, out, stat, *args, rest=rest)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            pyg.global_attention(*dev, *args, out=out, stat=stat, rest=rest)
            grads = pyg.global_attention_backward(gd, *dev, out, stat, *args, rest=rest)
        for _ in range(3):
            out.zero_()
            for t in grads:
                t.fill_(1)
            run(pyg, q, k, v, grad, table, lut, qn, kn, True)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for name, t in zip(("out", "grad_q", "grad_k", "grad_v", "grad_table"), (out, *grads)):
                assert torch.equal(t, first[name]), name


def test_empty_batches(pyg):
    z = torch.zeros(0, 2, 8, device="cuda")
    assert pyg.global_attention(z, z, z, torch.zeros(1, dtype=torch.int64, device="cuda")).shape == (0, 2, 8)
    x = torch.randn(5, 2, 8, device="cuda")
    out = pyg.global_attention(x, x, x, torch.zeros(1, dtype=torch.int64, device="cuda"))  # no graphs: no row has one
    assert (out == 0).all()
    ptr = torch.zeros(4, dtype=torch.int64, device="cuda")
    t = torch.ones(4, 2, device="cuda").requires_grad_(True)
    leaf = z.clone().requires_grad_(True)
    out = pyg.GlobalAttention.apply(leaf, z, z, t, ptr, None, pyg.relative_buckets(4, 8))
    gt, = torch.autograd.grad(out, [t], z)
    assert (gt == 0).all()


def test_refusals(pyg):
    x = torch.randn(6, 4, 8, device="cuda")
    ptr = ptr_of([6])
    ok = dict(q=x, k=x, v=x, ptr=ptr)
    lut, table = pyg.relative_buckets(8, 16), torch.zeros(8, 4, device="cuda")
    bad = [dict(q=x.half()), dict(q=x.cpu()), dict(q=x[0]), dict(k=x[:, :3], v=x[:, :3]), dict(v=x[:, :2]),
           dict(k=x[:5], v=x[:5]), dict(k=x.bfloat16(), v=x.bfloat16()), dict(q=x.transpose(1, 2)), dict(ptr=ptr.int()),
           dict(k_ptr=ptr_of([3, 3])), dict(table=table), dict(buckets=lut), dict(table=table[:, :2].contiguous(), buckets=lut),
           dict(table=table.bfloat16(), buckets=lut), dict(table=table, buckets=lut[1:]), dict(table=table, buckets=lut.long()),
           dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=1e-31), dict(out=x[:3]), dict(out=x.bfloat16()),
           dict(stat=torch.zeros(6, 4, device="cuda")), dict(rest=x)]
    for change in bad:
        with pytest.raises(ValueError):
            pyg.global_attention(**{**ok, **change})
    with pytest.raises(TypeError):
        pyg.global_attention([1], x, x, ptr)
    wide = torch.zeros(6, 1, 129, device="cuda")
    with pytest.raises(pyg.PygError):
        pyg.global_attention(wide, wide, wide, ptr)
    far = torch.zeros(2 * 1025 + 1, dtype=torch.int32, device="cuda")
    with pytest.raises(pyg.PygError):
        pyg.global_attention(x, x, x, ptr, None, table, far)
    with pytest.raises(pyg.PygError):
        pyg.global_attention(x, x, x, ptr, out=x)  # over its own input
    same = x[:1].expand(6, 4, 8)  # one row six times: rows overlap
    with pytest.raises(pyg.PygError):
        pyg.global_attention(x, same, same, ptr)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [8, 16, 24, 80, 128])
def test_few_queries_infinite_keys(pyg, D, dtype):
    """A key whose score is -infinity counts for nothing, whatever width its features are padded to: the
    result is that of the keys without it. One query a graph, in one range of keys and in several."""
    for qn, kn in (([1, 1], [40, 300]), ([1], [5000])):
        q, k, v, _, _, _ = inputs(11, qn, kn, 4, 2, D, DT[dtype], 0, 0, False, pyg)
        q[:, :, 0] = q[:, :, 0].abs() + 0.5
        at = [0, 7, sum(kn) - 1] + ([39, 40] if len(kn) > 1 else [])  # the first and last keys of the graphs too
        k[at, :, 0] = -math.inf
        keep = torch.ones(sum(kn), dtype=torch.bool)
        keep[at] = False
        left = [int(n.sum()) for n in keep.split(kn)]
        out = pyg.global_attention(q.cuda(), k.cuda(), v.cuda(), ptr_of(qn), ptr_of(kn))
        close({"out": out}, attention(q, k[keep], v[keep], qn, left), f"{D} {dtype} {kn}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [16, 24, 128])
def test_few_queries_infinite_values(pyg, D, dtype):
    """An infinite feature of the last key's value makes that feature of the result infinite, and no other."""
    for qn, kn in (([1, 1], [37, 301]), ([1], [5001])):
        q, k, v, _, _, _ = inputs(12, qn, kn, 4, 2, D, DT[dtype], 0, 0, False, pyg)
        ref = attention(q, k, v, qn, kn)
        v[sum(kn) - 1, 1, 3] = math.inf  # key head 1: query heads 2 and 3
        out = pyg.global_attention(q.cuda(), k.cuda(), v.cuda(), ptr_of(qn), ptr_of(kn)).cpu()
        assert (out[-1, 2:, 3] == math.inf).all(), out[-1, 2:, 3]
        out[-1, 2:, 3] = ref["out"][0][-1, 2:, 3].to(out.dtype)
        close({"out": out}, ref, f"{D} {dtype} {kn}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("qn,kn,causal", [([20, 31, 5], None, False), ([70, 33], [90, 120], True), ([300, 150], None, False), ([200], [330], True)])
def test_every_offset_has_its_bucket(pyg, qn, kn, causal, dtype):
    """A bucket for every offset: each of the table's gradients is the sum of one diagonal, and those beyond the
    reach the sum of the corners, over several tiles of a wavefront and several wavefronts."""
    same = kn is None
    kn = qn if same else kn
    for reach in (3, 40, 100):
        q, k, v, grad, _, _ = inputs(13, qn, kn, 3, 1, 24, DT[dtype], 0, 0, causal, pyg)
        table = torch.randn(2 * reach + 1, 3, generator=torch.Generator().manual_seed(reach)).to(DT[dtype])
        lut = torch.arange(2 * reach + 1, dtype=torch.int32)
        got = run(pyg, q, k, v, grad, table, lut, qn, kn, causal, same=same)
        close(got, attention(q, k, v, qn, kn, table, lut, causal, grad=grad), f"{reach} {dtype}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("qn,kn,H,Hkv,causal", [([1100], [4500], 2, 1, True), ([1300, 5], [5000, 1200], 1, 1, False)])
def test_many_queries_over_a_longer_history(pyg, qn, kn, H, Hkv, causal, dtype):
    """More than 1,024 queries a graph whose keys are still cut into ranges in the backward."""
    q, k, v, grad, table, lut = inputs(14, qn, kn, H, Hkv, 16, DT[dtype], 8, 64, causal, pyg)
    got = run(pyg, q, k, v, grad, table, lut, qn, kn, causal)
    close(got, attention(q, k, v, qn, kn, table, lut, causal, grad=grad), f"{qn} {dtype}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("qn,kn", [([1, 2], [2500, 2000]), ([20, 45], [50, 90]), ([150, 3], [200, 130])])
def test_gradients_that_are_not_wanted(pyg, qn, kn, dtype):
    """Each set of wanted gradients is what the whole call gives of it, to the bit, with rows of no graph behind."""
    q, k, v, grad, table, lut = (t.cuda() for t in inputs(15, qn, kn, 4, 2, 32, DT[dtype], 8, 16, True, pyg, extra=3))
    stat = torch.empty((*q.shape[:2], 2), device="cuda")
    args = (ptr_of(qn), ptr_of(kn), table, lut, True)
    out = pyg.global_attention(q, k, v, *args, stat=stat)
    whole = pyg.global_attention_backward(grad, q, k, v, out, stat, *args)
    for wanted in range(8):
        a, b, c = bool(wanted & 1), bool(wanted & 2), bool(wanted & 4)
        got = pyg.global_attention_backward(grad, q, k, v, out, stat, *args, need_grad_q=a, need_grad_kv=b, need_grad_table=c)
        for x, y, need in zip(got, whole, (a, b, b, c)):
            assert torch.equal(x, y) if need else x is None
    for i in range(4):  # and through autograd
        leaves = [t.clone().requires_grad_(i == j) for j, t in enumerate((q, k, v, table))]
        out = pyg.GlobalAttention.apply(*leaves, args[0], args[1], lut, True)
        got, = torch.autograd.grad(out, [leaves[i]], grad)
        full = [t.clone().requires_grad_(True) for t in (q, k, v, table)]
        out = pyg.GlobalAttention.apply(*full, args[0], args[1], lut, True)
        assert torch.equal(got, torch.autograd.grad(out, full, grad)[i])


@pytest.mark.parametrize("D", [1, 8])
def test_broadcast_inputs(pyg, D):
    """One row or head that stands for all of them: the gradient of the small tensor is the sum."""
    n, H = [9, 40], 4
    g = torch.Generator().manual_seed(16)
    grad = torch.randn(sum(n), H, D, generator=g)
    small = [torch.randn(sum(n), 1, D, generator=g), torch.randn(1, H, D, generator=g), torch.randn(sum(n), 1, D, generator=g)]
    whole = [t.expand(sum(n), H, D) for t in small]
    ref = attention(*whole, n, n, grad=grad)
    leaves = [t.cuda().requires_grad_(True) for t in small]
    out = pyg.GlobalAttention.apply(*[t.expand(sum(n), H, D) for t in leaves], None, ptr_of(n))
    grads = torch.autograd.grad(out, leaves, grad.cuda())
    close({"out": out}, ref, "out")
    for name, got, dim in zip(("grad_q", "grad_k", "grad_v"), grads, (1, 0, 1)):
        val, bound = (t.sum(dim, keepdim=True) for t in ref[name])  # and the sum in fp32 of so many terms
        close({name: got}, {name: (val, bound + sum(n) * 2.0 ** -24 * ref[name][0].abs().sum(dim, keepdim=True))}, "broadcast")
