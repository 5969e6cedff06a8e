"""The attention kernels' forms one by one: inputs that reach each of them (few queries in
one range of keys and in several, lone wavefronts, workgroups of four, heads of a group dealt out)
with rows of no graph, with poisoned neighbours, and with what the forward hands the backward
beside its result pinned by itself."""
import math

import pytest
import torch

from tests.attention_reference import U32, attention, close
from tests.test_global_attention_gpu import DT, inputs, ptr_of, pyg, run  # noqa: F401 (pyg is the fixture)

pytestmark = pytest.mark.gpu


# Backward: workgroups of four wavefronts (more than 1,024 queries a graph on average, or many heads), with the heads
# of a group dealt out over workgroups where they are shared.
FOUR = [
    ([1100], None, 2, 2, 64, 32, 24, False),
    ([1500, 700], None, 4, 1, 32, 16, 64, True),
    ([1100], [1300], 3, 1, 40, 8, 8, True),
    ([1300], [1100], 6, 2, 128, 32, 128, False),
    ([1030], None, 2, 1, 128, 8, 16, True),
    ([1025], None, 1, 1, 16, 64, 100, False),
    ([1090], None, 1, 1, 1, 0, 0, False),
    ([1060], None, 1, 1, 128, 1024, 1024, False),
    ([300, 1, 200], None, 160, 10, 8, 4, 4, True),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("i", range(len(FOUR)))
def test_large_graphs(pyg, i, dtype):  # noqa: F811
    qn, kn, H, Hkv, D, buckets, reach, causal = FOUR[i]
    same = kn is None
    kn = qn if same else kn
    q, k, v, grad, table, lut = inputs(100 + i, qn, kn, H, Hkv, D, DT[dtype], buckets, reach, causal, pyg)
    got = run(pyg, q, k, v, grad, table, lut, qn, kn, causal, same=same)
    close(got, attention(q, k, v, qn, kn, table, lut, causal, grad=grad), f"case {i} {dtype}")


PADDED = [  # queries, keys, heads, key heads, features, rows of no graph
    ([1] * 8, [40] * 8, 2, 2, 16, 20),            # 16-row tiles, one range
    ([1, 2], [3000, 2000], 4, 2, 24, 20),         # several ranges, forward and dQ
    ([20, 30], [20, 30], 2, 2, 16, 13),           # lone wavefronts
    ([1100], [1000], 2, 2, 16, 150),              # four wavefronts
    ([900], [900], 40, 10, 8, 100),               # and heads of a group over several workgroups
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("i", range(len(PADDED)))
def test_rows_of_no_graph_in_every_form(pyg, i, dtype):  # noqa: F811
    """Zeros in results made here, whatever the workspace held; a caller's result left alone."""
    qn, kn, H, Hkv, D, extra = PADDED[i]
    q, k, v, grad, table, lut = inputs(200 + i, qn, kn, H, Hkv, D, DT[dtype], 8, 16, False, pyg, extra=extra)
    n, m = sum(qn), sum(kn)
    q[n:], k[m:], v[m:], grad[n:] = (math.nan,) * 4
    ref = attention(q[:n], k[:m], v[:m], qn, kn, table, lut, False, grad=grad[:n])
    dev = [t.cuda() for t in (q, k, v)]
    args = (ptr_of(qn), ptr_of(kn), table.cuda(), lut.cuda())
    ws = torch.full((1 << 26,), math.nan, device="cuda")
    stat = torch.full((*q.shape[:2], 2), math.nan, device="cuda")
    rest = torch.full(q.shape, math.nan, dtype=q.dtype, device="cuda") if dtype == "bf16" else None
    out = pyg.global_attention(*dev, *args, stat=stat, rest=rest, workspace=ws)
    ws.fill_(math.nan)
    grads = pyg.global_attention_backward(grad.cuda(), *dev, out, stat, *args, rest=rest, workspace=ws)
    for name, t, rows in zip(("out", "grad_q", "grad_k", "grad_v", "grad_table"), (out, *grads), (n, n, m, m, len(table))):
        assert (t[rows:] == 0).all(), name
        close({name: t[:rows]}, ref, f"form {i} {dtype}")
    mine = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    pyg.global_attention(*dev, *args, out=mine, workspace=ws)
    assert (mine[n:] == 7).all() and torch.equal(mine[:n], out[:n])


@pytest.mark.parametrize("qn,kn", [([1, 2, 1], [40, 300, 60]), ([1, 2, 1], [3000, 2500, 2000]), ([1050, 1100, 1000], None)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_leak_between_graphs_in_every_form(pyg, qn, kn, dtype):  # noqa: F811
    """NaN and infinities in one graph change nothing of its neighbours, which share its tiles and ranges."""
    same = kn is None
    kn = qn if same else kn
    q, k, v, grad, table, lut = inputs(300, qn, kn, 2, 1, 24, DT[dtype], 8, 16, False, pyg)
    clean = run(pyg, q, k, v, grad, table, lut, qn, kn, False, same=same)
    for t, n in ((q, qn), (grad, qn), (k, kn), (v, kn)):
        t[n[0]:n[0] + n[1]] = math.inf
        t[n[0]] = math.nan
    bad = run(pyg, q, k, v, grad, table, lut, qn, kn, False, same=same)
    for name, n in (("out", qn), ("grad_q", qn), ("grad_k", kn), ("grad_v", kn)):
        a, b = n[0], n[0] + n[1]
        assert torch.equal(bad[name][:a], clean[name][:a]) and torch.equal(bad[name][b:], clean[name][b:]), name
        assert not torch.isfinite(bad[name][a:b]).all()


REST = [  # queries, keys, causal: every form of the forward and of dQ
    ([1, 2], [37, 300], False),
    ([1], [600], False),
    ([3], [1030], True),
    ([33, 20, 60], [33, 20, 60], True),
    ([200, 129], [200, 129], False),
    ([1100], [40], False),
]


def flat(qn, kn, causal):
    """Inputs whose rows weigh all the keys they see alike (q is 0), with values far from 0 beside their spread, and
    the weights: P is 1 / n, its parts in bf16 exact, so that nothing but the result's own rounding is lost."""
    g = torch.Generator().manual_seed(17)
    H, D = 2, 8
    q = torch.zeros(sum(qn), H, D).bfloat16()
    k, v = ((torch.randn(sum(kn), H, D, generator=g) * s + o).bfloat16() for s, o in ((1, 4), (0.25, 16)))
    grad = torch.randn(sum(qn), H, D, generator=g).bfloat16()
    P = torch.zeros(sum(qn), sum(kn), dtype=torch.float64)
    i0 = j0 = 0
    for n, m in zip(qn, kn):
        seen = torch.arange(m)[None] <= torch.arange(m - n, m)[:, None] if causal else torch.ones(n, m, dtype=torch.bool)
        P[i0:i0 + n, j0:j0 + m] = seen / seen.sum(1, keepdim=True).clamp(min=1)
        i0, j0 = i0 + n, j0 + m
    return q, k, v, grad, P


@pytest.mark.parametrize("qn,kn,causal", REST)
def test_rest_is_what_rounding_took(pyg, qn, kn, causal):  # noqa: F811
    """out + rest is the result to 8 bits more than out: the mean of the values. It is off by
    rest's own rounding, half a step (2^-8) of at most half a step of the result, by a sum of n terms and its division."""
    q, k, v, _, P = flat(qn, kn, causal)
    rest = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    out = pyg.global_attention(q.cuda(), k.cuda(), v.cuda(), ptr_of(qn), ptr_of(kn), causal=causal, rest=rest).cpu().double()
    rest = rest.cpu().double()
    want = torch.einsum("ij,jhd->ihd", P, v.double())
    bound = ((max(kn) + 4) * U32 + 2.0 ** -16) * 1.01 * want.abs()  # the magnitudes' mean: values are positive
    assert (v > 0).all() and ((out + rest - want).abs() <= bound).all()
    for wrong in (0.0, -1.0):
        assert ((out + wrong * rest - want).abs() > bound).any()


@pytest.mark.parametrize("qn,kn,causal", REST)
def test_rest_reaches_the_gradients(pyg, qn, kn, causal):  # noqa: F811
    """delta_i = <g_i, out_i + rest_i>: dS = P (dP - delta) cancels, and out's rounding alone would be most of what is left.
    Bounds as in the general reference, with delta's error that of out + rest; without rest, and with it the wrong
    way round, grad_q lies outside them (and the table's gradient, where it is the sum of few rows and keys)."""
    q, k, v, grad, P = flat(qn, kn, causal)
    H, D = q.shape[1:]
    c, n, half = D ** -0.5, max(kn), torch.finfo(torch.bfloat16).eps / 2
    table, lut = torch.zeros(4, H).bfloat16(), pyg.relative_buckets(4, 8, True, "cpu")
    R = len(lut) // 2
    g, x, y = grad.double(), k.double(), v.double()
    o = torch.einsum("ij,jhd->ihd", P, y)
    dp = torch.einsum("ihd,jhd->hij", g, y)
    mag = torch.einsum("ihd,jhd->hij", g.abs(), y.abs())
    delta = (g * o).sum(2).T[:, :, None]
    derr = (g.abs() * o.abs()).sum(2).T[:, :, None] * (2.0 ** -16 * 1.01 + (n + 4 + D + 2) * U32)
    ds = P * (dp - delta)
    dserr = P * ((n + 16) * U32 * (dp - delta).abs() + (D + 2) * U32 * mag + derr)
    dsr = dserr + half * (ds.abs() + dserr)
    want = {"grad_q": c * torch.einsum("hij,jhd->ihd", ds, x)}
    bound = {"grad_q": c * torch.einsum("hij,jhd->ihd", dsr + (n + 2) * U32 * ds.abs(), x.abs())}
    i0 = j0 = 0
    idx = torch.full(P.shape, -1)
    for a, b in zip(qn, kn):
        off = torch.arange(b)[None] - torch.arange(b - a, b)[:, None]
        idx[i0:i0 + a, j0:j0 + b] = lut.long()[off.clamp(-R, R) + R]
        i0, j0 = i0 + a, j0 + b
    want["grad_table"], bound["grad_table"] = (torch.stack([torch.stack([(t[h] * (idx == b)).sum() for h in range(H)]) for b in range(4)])
                                               for t in (ds, dserr + (n + sum(qn) + 64) * U32 * ds.abs()))
    for name in want:
        bound[name] = bound[name] + half * (want[name].abs() + bound[name]) + 1e-30
    dev = [t.cuda() for t in (q, k, v)]
    args = (ptr_of(qn), ptr_of(kn), table.cuda(), lut.cuda(), causal)
    stat, rest = torch.empty(*q.shape[:2], 2, device="cuda"), torch.empty(q.shape, dtype=q.dtype, device="cuda")
    out = pyg.global_attention(*dev, *args, stat=stat, rest=rest)

    def off(r):
        got = pyg.global_attention_backward(grad.cuda(), *dev, out, stat, *args, rest=r)
        return {name: float(((t.cpu().double() - want[name]).abs() / bound[name]).max()) for name, t in (("grad_q", got[0]), ("grad_table", got[3]))}
    right = off(rest)
    assert all(e <= 1 for e in right.values()), right
    for wrong in (None, -rest):
        e = off(wrong)
        assert e["grad_q"] > 1 and (sum(qn) > 3 or max(kn) > 600 or e["grad_table"] > 1), e


def test_captured_with_a_workspace_that_others_write(pyg):  # noqa: F811
    """A captured call brings its own workspace and reads nothing that an earlier replay left in it."""
    for qn, kn, D in (([1, 1], [3000, 1100], 128), ([1100], [1100], 64)):
        q, k, v, grad, table, lut = (t.cuda() for t in inputs(18, qn, kn, 4, 2, D, torch.bfloat16, 32, 64, True, pyg))
        args = (ptr_of(qn), ptr_of(kn), table, lut, True)
        stat, rest, out = torch.empty(*q.shape[:2], 2, device="cuda"), torch.empty_like(q), torch.empty_like(q)
        ws = torch.zeros(1 << 26, device="cuda")

        def call():
            pyg.global_attention(q, k, v, *args, out=out, stat=stat, rest=rest, workspace=ws)
            return pyg.global_attention_backward(grad, q, k, v, out, stat, *args, rest=rest, workspace=ws)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            want = [t.clone() for t in (*call(), out)]
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            grads = call()
        for fill in (math.nan, 1.0, math.inf):
            for t in (ws, stat, rest, out, *grads):
                t.fill_(fill)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip((*grads, out), want))


HIDDEN = [  # queries, keys, heads, key heads, features: every form, causal
    ([2, 5], [40, 300], 2, 1, 24),
    ([1], [600], 2, 2, 32),
    ([2, 3], [1100, 2050], 2, 1, 128),
    ([33, 20, 70], None, 2, 1, 16),
    ([40, 90], [70, 60], 2, 2, 80),
    ([300, 200], None, 2, 1, 64),
    ([260], None, 2, 1, 128),
    ([1100], [1150], 2, 1, 32),
    ([1040], None, 2, 1, 128),
    ([1100], None, 1, 1, 64),
    ([30, 45], None, 2, 1, 7),
    ([3], [70], 2, 2, 33),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("i", range(len(HIDDEN)))
def test_what_a_row_does_not_see_may_be_anything(pyg, i, dtype):  # noqa: F811
    """NaN and infinities in a key, value, query or gradient reach what sees them and nothing else: results in
    which they have no part are those of clean inputs, the rows in which they have one are not finite."""
    qn, kn, H, Hkv, D = HIDDEN[i]
    same = kn is None
    kn = qn if same else kn
    reach = 6
    q, k, v, grad, _, _ = inputs(400 + i, qn, kn, H, Hkv, D, DT[dtype], 0, 0, True, pyg)
    lut = torch.arange(2 * reach + 1, dtype=torch.int32)  # a bucket for every offset, the later keys' unused
    table = torch.randn(2 * reach + 1, H, generator=torch.Generator().manual_seed(i)).to(DT[dtype])
    M = torch.zeros(sum(qn), sum(kn), dtype=torch.bool)  # whether query i sees key j
    i0 = j0 = 0
    for n, m in zip(qn, kn):
        M[i0:i0 + n, j0:j0 + m] = torch.arange(m)[None] <= torch.arange(m - n, m)[:, None]
        i0, j0 = i0 + n, j0 + m
    ref = attention(q, k, v, qn, kn, table, lut, True, grad=grad)

    def call(q, k, v, g):
        got = run(pyg, q, k, v, g, table, lut, qn, kn, True, same=same)
        assert (got["grad_table"][reach + 1:] == 0).all()  # offsets that no row sees
        return {n: t.cpu() for n, t in got.items()}

    def others(got, x, part, what):
        close({x: got[x][~part]}, {x: tuple(t[~part] for t in ref[x])}, str(what))

    def odd(t):
        return not torch.isfinite(t).all(2).any()
    clean = call(q, k, v, grad)
    close(clean, ref, "clean")
    for j in (kn[0] - 1, max(kn[0] - 3, 0), sum(kn) - 1 - kn[-1] // 2):
        rows = M[:, j]
        beside = M[rows].any(0)  # keys seen by a row that sees key j
        for value in ("k", math.nan, math.inf, -math.inf):
            bad_k, bad_v = k.clone(), v.clone()
            if value == "k":
                bad_k[j, :, 1] = math.nan
            else:
                bad_v[j, :, 1] = value
            got = call(q, bad_k, bad_v, grad)
            for x, part in (("out", rows), ("grad_q", rows), ("grad_k", beside), ("grad_v", beside & (value == "k"))):
                others(got, x, part, (value, j))
            assert odd(got["out"][rows]) and odd(got["grad_q"][rows]) and odd(got["grad_k"][beside])
    for r in (min(2, qn[0] - 1), sum(qn) - 1 - qn[-1] // 2):
        rows, keys = torch.arange(sum(qn)) == r, M[r]
        for value in ("q", math.nan, math.inf):
            bad_q, bad_g = q.clone(), grad.clone()
            if value == "q":
                bad_q[r, :, 1] = math.nan
            else:
                bad_g[r, :, 1] = value
            got = call(bad_q, k, v, bad_g)
            sees = rows & bool(keys.any())  # a row that sees nothing has zeros whatever it holds
            for x, part in (("out", sees & (value == "q")), ("grad_q", sees), ("grad_k", keys), ("grad_v", keys)):
                others(got, x, part, (value, r))
            assert odd(got["grad_q"][sees]) and odd(got["grad_k"][keys]) and odd(got["grad_v"][keys])
    # and all of it at once, which ends
    nan = [torch.full_like(t, math.nan) for t in (q, k, v, grad)]
    got = call(*nan)
    assert odd(got["out"][M.any(1)]) and odd(got["grad_q"][M.any(1)]) and odd(got["grad_k"][M.any(0)]) and odd(got["grad_v"][M.any(0)])


@pytest.mark.parametrize("qn,kn,causal", [([2], [700], False), ([3, 33], [1100, 3000], True), ([40, 90], [90, 60], False), ([300], [310], True),
                                          ([1060], None, False)])
@pytest.mark.parametrize("low", [-1e5, 3e4])
def test_biases_far_larger_than_the_products(pyg, qn, kn, causal, low):  # noqa: F811
    """fp32 products are summed by themselves and the bias added once: a bias that all keys share costs one
    rounding at its magnitude and not one of every partial sum of 128 features (the reference's bound
    allows four)."""
    same = kn is None
    kn = qn if same else kn
    q, k, v, grad, table, lut = inputs(500, qn, kn, 2, 1, 128, torch.float32, 4, 12, causal, pyg)
    table[:] = low
    got = run(pyg, q, k, v, grad, table, lut, qn, kn, causal, same=same)
    close(got, attention(q, k, v, qn, kn, table, lut, causal, grad=grad), f"{low} {qn}")
