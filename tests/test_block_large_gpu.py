"""The transformer block's operators on arrays of more than 2^31 elements: the last rows, whose offsets no longer fit
32 bits, come out as they do by themselves."""
import pytest
import torch

pytestmark = [pytest.mark.gpu, pytest.mark.slow]
N, F, GRAPH = 17_000_000, 128, 100  # 2.18e9 elements
LAST = 50 * GRAPH


@pytest.fixture(scope="module")
def pyg():
    import paper_1903_02428_amd as m
    assert torch.cuda.is_available()
    m.library()
    return m


@pytest.fixture
def rows():
    """A function that makes [N, F] bf16 rows, zeros but for the last ones; they are freed after the test."""
    g = torch.Generator(device="cuda").manual_seed(0)

    def make():
        t = torch.zeros(N, F, dtype=torch.bfloat16, device="cuda")
        t[-LAST:] = torch.randn(LAST, F, device="cuda", generator=g)
        return t
    yield make
    torch.cuda.empty_cache()


def test_attention_of_many_graphs(pyg, rows):
    q, k, v, g = (rows().view(N, 1, F) for _ in range(4))
    ptr = torch.arange(0, N + 1, GRAPH, device="cuda")
    table, lut = torch.randn(8, 1, device="cuda").bfloat16(), pyg.relative_buckets(8, 16)
    end, few = [t[-LAST:].contiguous() for t in (q, k, v, g)], torch.arange(0, LAST + 1, GRAPH, device="cuda")

    def call(q, k, v, g, ptr):
        stat, rest = torch.empty(q.shape[0], 1, 2, device="cuda"), torch.empty_like(q)
        out = pyg.global_attention(q, k, v, ptr, None, table, lut, True, stat=stat, rest=rest)
        return (out, *pyg.global_attention_backward(g, q, k, v, out, stat, ptr, None, table, lut, True, rest=rest)[:3])
    for name, got, want in zip(("out", "grad_q", "grad_k", "grad_v"), call(q, k, v, g, ptr), call(*end, few)):
        assert torch.equal(got[-LAST:], want), name
        assert (got[:LAST] == 0).all(), name


def test_one_query_over_a_long_history(pyg, rows):
    """Keys that weigh nothing (their score is about 60 below) ahead of the last ones, causal."""
    k, v = rows().view(N, 1, F), rows().view(N, 1, F)
    k[:, 0, 0] = -60.0
    k[-LAST:, 0, 0] = 0.0
    q = torch.randn(1, 4, F, device="cuda").bfloat16()
    q[:, :, 0] = F ** 0.5
    g = torch.randn(1, 4, F, device="cuda").bfloat16()

    def call(k, v):
        ptr, k_ptr = torch.tensor([0, 1], device="cuda"), torch.tensor([0, len(k)], device="cuda")
        stat = torch.empty(1, 4, 2, device="cuda")
        out = pyg.global_attention(q, k, v, ptr, k_ptr, causal=True, stat=stat)
        return (out, *pyg.global_attention_backward(g, q, k, v, out, stat, ptr, k_ptr, causal=True)[:3])
    for name, got, want in zip(("out", "grad_q", "grad_k", "grad_v"), call(k, v), call(k[-LAST:], v[-LAST:])):
        got = got[-LAST:] if len(got) > 1 else got
        # sums of 5,000 terms in other ranges, each weight and result rounded to bf16
        err = (got.double() - want.double()).norm() / want.double().norm()
        assert err <= 4 * 2.0 ** -8, (name, float(err))


def test_norms_checkpoints_and_dense_gradients(pyg, rows):
    h, r, g = rows(), rows(), rows()
    w = torch.randn(F, device="cuda")
    end = [t[-LAST:].contiguous() for t in (h, r, g)]

    def norm(h, r, g):
        s, y, kept = pyg.block_norm(h, r, post_weight=w, weight=w, bias=w, norm="rms", checkpoint=True)
        grads = pyg.block_norm_backward(g, g, h, r, post_weight=w, weight=w, bias=w, norm="rms",
                                        need=(True, True) + (False,) * 6)
        return s, y, kept.codes, kept.steps, *grads[:2]
    for a, b in zip(norm(h, r, g), norm(*end)):
        assert torch.equal(a[-LAST:], b)
    kept, small = pyg.activation_checkpoint(h), pyg.activation_checkpoint(end[0])
    assert torch.equal(kept.codes[-LAST:], small.codes) and torch.equal(kept.steps[-LAST:], small.steps)
    assert torch.equal(pyg.checkpoint_restore(kept)[-LAST:], pyg.checkpoint_restore(small))
    theta = torch.randn(F, F, device="cuda").bfloat16()
    gx, gt = pyg.dense_transform_backward(g, theta, kept)
    sx, st = pyg.dense_transform_backward(end[2], theta, small)
    assert torch.equal(gx[-LAST:], sx) and (gx[:LAST] == 0).all()
    # the same 5,000 products in another order
    bound = (LAST + 8) * 2.0 ** -24 * (pyg.checkpoint_restore(small, torch.float32).abs().T @ end[2].float().abs())
    assert ((gt.float() - st.float()).abs() <= bound + 2.0 ** -7 * st.float().abs()).all()
