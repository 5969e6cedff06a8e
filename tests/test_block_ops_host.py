"""The transformer block's C entries without a GPU: bad arguments are refused on the
host before any device work, and workspace queries answer for what is allowed."""
import ctypes
import os

import pytest

PYG_OK, INVALID, WORKSPACE, UNSUPPORTED = 0, -1, -3, -5
A, B_, C_, D_ = (ctypes.c_void_p(0x100000 * i) for i in (1, 2, 3, 4))  # never dereferenced


@pytest.fixture(scope="module")
def lib():
    import paper_1903_02428_amd as pyg
    if not os.path.exists(pyg.library_path()):
        from paper_1903_02428_amd import build
        build.build()
    return pyg.library()


def attention(**change):
    from paper_1903_02428_amd.binding import _Attention
    a = dict(q_ptr=0x1000, k_ptr=0x1000, B=2, Nq=100, Nk=100, H=4, Hkv=2, D=32, q_row=128, q_head=32, k_row=64, k_head=32,
             v_row=64, v_head=32, dtype=1, scale=0.2, causal=0, table=0x2000, bucket=0x3000, buckets=8, reach=16, zero_rest=1)
    a.update(change)
    return _Attention(*a.values())


def size(fn, *args):
    out = ctypes.c_size_t(0)
    return fn(*args, ctypes.byref(out)), out.value


def test_attention_refusals(lib):
    def rc(a, q=A, out=D_, stat=None, rest=None, ws=A, nbytes=1 << 40):
        return lib.pyg_global_attention(ctypes.byref(a) if a else None, q, B_, C_, out, stat, rest, ws, nbytes, None)
    assert rc(None) == INVALID
    for change in (dict(dtype=7), dict(B=-1), dict(Nq=-1), dict(H=0), dict(Hkv=3), dict(D=0), dict(scale=0.0), dict(scale=-1.0),
                   dict(scale=float("nan")), dict(scale=float("inf")), dict(bucket=None), dict(buckets=0), dict(reach=-1),
                   dict(q_ptr=None), dict(k_ptr=None), dict(q_row=0), dict(k_head=0), dict(v_row=32), dict(q_head=64)):
        assert rc(attention(**change)) == INVALID, change
    for change in (dict(D=129, q_head=129, q_row=600, k_head=129, k_row=300, v_head=129, v_row=300), dict(reach=1025), dict(buckets=1025),
                   dict(Nq=1 << 31), dict(H=65536), dict(q_row=1 << 22)):
        assert rc(attention(**change)) == UNSUPPORTED, change
    assert rc(attention(), q=None) == INVALID and rc(attention(), out=None) == INVALID
    assert rc(attention(dtype=0), rest=A) == INVALID  # nothing is rounded away in fp32
    few = attention(Nq=2, Nk=100_000)
    status, need = size(lib.pyg_global_attention_workspace, ctypes.byref(few))
    assert status == PYG_OK and need >= 2 * 4 * (32 + 2) * 4
    assert rc(few, nbytes=need - 1) == WORKSPACE and rc(few, ws=None) == WORKSPACE
    assert size(lib.pyg_global_attention_workspace, ctypes.byref(attention(Nq=0))) == (PYG_OK, 0)
    assert rc(attention(Nq=0), q=None, out=None) == PYG_OK  # nothing to do


def test_attention_backward_refusals(lib):
    a = attention()
    status, need = size(lib.pyg_global_attention_backward_workspace, ctypes.byref(a))
    assert status == PYG_OK and need >= 100 * 4 * 4

    def rc(a=a, **change):
        p = dict(g=A, q=A, k=B_, v=C_, out=A, stat=A, rest=None, gq=D_, gk=D_, gv=D_, gt=D_, ws=A, n=need)
        p.update(change)
        return lib.pyg_global_attention_backward(ctypes.byref(a), *p.values(), None)
    for name in ("g", "q", "k", "v", "out", "stat", "gq", "gk", "gv"):
        assert rc(**{name: None}) == INVALID, name
    assert rc(attention(table=None), gt=D_) == INVALID
    assert rc(n=need - 1) == WORKSPACE and rc(ws=None) == WORKSPACE


def norm(**change):
    from paper_1903_02428_amd.binding import _BlockNorm
    a = dict(dtype=0, norm=0, N=10, F=64, eps=1e-5, h=0x1000, residual=0x2000, gate=None, gate_rows=0, scale=0x3000, post_weight=0x4000,
             post_bias=0x5000, weight=0x6000, bias=0x7000)
    a.update(change)
    return _BlockNorm(*a.values())


def test_block_norm_refusals(lib):
    def rc(a, r=A, y=B_, codes=None, steps=None):
        return lib.pyg_block_norm(ctypes.byref(a), r, y, codes, steps, None)
    for change in (dict(dtype=3), dict(norm=2), dict(N=-1), dict(F=0), dict(eps=-1.0), dict(eps=float("nan")), dict(post_weight=None),
                   dict(weight=None), dict(h=None)):
        assert rc(norm(**change)) == INVALID, change
    assert rc(norm(F=8193)) == UNSUPPORTED and rc(norm(N=1 << 31)) == UNSUPPORTED
    assert rc(norm(), y=None) == INVALID and rc(norm(weight=None, bias=None), y=B_) == INVALID
    assert rc(norm(), codes=A) == INVALID and rc(norm(weight=None, bias=None), y=None, codes=A, steps=B_) == INVALID
    assert rc(norm(N=0), r=None, y=None) == PYG_OK
    status, need = size(lib.pyg_block_norm_backward_workspace, ctypes.byref(norm()))
    assert status == PYG_OK and need > 0

    def back(a=norm(), gr=A, gy=B_, gate=None, scale=D_, n=need, ws=A):
        return lib.pyg_block_norm_backward(ctypes.byref(a), gr, gy, C_, C_, gate, scale, D_, D_, D_, D_, ws, n, None)
    assert back(gr=None, gy=None) == INVALID and back(gate=D_) == INVALID and back(norm(scale=None)) == INVALID
    assert back(norm(weight=None, bias=None)) == INVALID
    assert back(n=need - 1) == WORKSPACE and back(ws=None) == WORKSPACE


def test_checkpoint_and_dense_refusals(lib):
    ck = lib.pyg_activation_checkpoint
    assert ck(A, 5, 4, 8, B_, C_, None) == INVALID and ck(A, 0, -1, 8, B_, C_, None) == INVALID and ck(A, 0, 4, 0, B_, C_, None) == INVALID
    assert ck(None, 0, 4, 8, B_, C_, None) == INVALID and ck(A, 0, 4, 8, ctypes.c_void_p(0x1004), C_, None) == INVALID
    assert ck(A, 0, 1 << 31, 8, B_, C_, None) == UNSUPPORTED and ck(None, 0, 0, 8, None, None, None) == PYG_OK
    assert lib.pyg_checkpoint_restore(A, B_, 4, 8, None, 0, None) == INVALID
    status, need = size(lib.pyg_dense_transform_backward_workspace, 0, 1000, 64, 32)
    assert status == PYG_OK and need >= 64 * 32 * 4
    assert size(lib.pyg_dense_transform_backward_workspace, 0, 1000, 0, 32)[0] == INVALID

    def rc(dtype=0, N=1000, Fo=32, Fi=64, g=A, theta=B_, codes=C_, gx=D_, gt=D_, ws=A, n=need):
        return lib.pyg_dense_transform_backward(g, dtype, N, Fo, theta, Fi, codes, C_, gx, gt, ws, n, None)
    assert rc(dtype=2) == INVALID and rc(g=None) == INVALID and rc(theta=None) == INVALID and rc(codes=None) == INVALID
    assert rc(codes=ctypes.c_void_p(0x1008)) == INVALID and rc(Fi=1 << 24) == UNSUPPORTED
    assert rc(n=need - 1) == WORKSPACE and rc(ws=None) == WORKSPACE


def test_relative_buckets():
    import paper_1903_02428_amd as pyg
    t = pyg.relative_buckets(8, 16, True, "cpu").tolist()
    assert t[16] == 0 and t[15] == 1 and t[17] == 5 and t[0] == 3 and t[-1] == 7  # own buckets for later keys
    assert sorted(set(t)) == [0, 1, 2, 3, 5, 6, 7]  # no later key at distance 0
    t = pyg.relative_buckets(8, 32, False, "cpu").tolist()
    assert t[33:] == [0] * 32 and t[:33][::-1] == sorted(t[:33]) and t[0] == 7
    for bad in ((1, 8, True), (8, 2, True), (7, 8, True), (0, 8, False)):
        with pytest.raises(ValueError):
            pyg.relative_buckets(*bad, "cpu")


def at(address):
    return ctypes.c_void_p(address)


def test_attention_overlaps(lib):
    """Results that share a byte with an input, another result or the workspace are refused; so
    every pair is, in both directions (nothing here reaches a device: the call ends at the check)."""
    M = 1 << 30
    few = attention(Nq=2, Nk=100_000)
    need = size(lib.pyg_global_attention_workspace, ctypes.byref(few))[1]
    base = dict(q=M, k=2 * M, v=3 * M, out=4 * M, stat=5 * M, rest=6 * M, ws=7 * M)
    last = dict(q=2 * 128 * 2 - 2, k=100_000 * 64 * 2 - 2, out=2 * 128 * 2 - 2, stat=2 * 4 * 8 - 4, rest=2 * 128 * 2 - 2,
                ws=need - 4)
    last["v"] = last["k"]

    def rc(p, a=few):
        return lib.pyg_global_attention(ctypes.byref(a), *[at(p[n]) for n in ("q", "k", "v", "out", "stat", "rest", "ws")], need, None)
    for r in ("out", "stat", "rest", "ws"):
        for o in base:
            if o != r:
                assert rc({**base, r: base[o]}) == INVALID, (r, o)
                assert rc({**base, r: base[o] + last[o]}) == INVALID, (r, o, "last")
                assert rc({**base, r: base[o] - last[r]}) == INVALID, (r, o, "first")
        for field in ("q_ptr", "k_ptr", "table", "bucket"):
            assert rc({**base, r: M // 2}, attention(Nq=2, Nk=100_000, **{field: M // 2})) == INVALID, (r, field)

    a = attention()
    need = size(lib.pyg_global_attention_backward_workspace, ctypes.byref(a))[1]
    names = ("g", "q", "k", "v", "out", "stat", "rest", "gq", "gk", "gv", "gt", "ws")
    base = {n: (i + 1) * M for i, n in enumerate(names)}

    def back(p, a=a):
        return lib.pyg_global_attention_backward(ctypes.byref(a), *[at(p[n]) for n in names], need, None)
    for r in ("gq", "gk", "gv", "gt", "ws"):
        for o in names:
            if o != r:
                assert back({**base, r: base[o]}) == INVALID and back({**base, r: base[o] + 60}) == INVALID, (r, o)
        for field in ("q_ptr", "k_ptr", "table", "bucket"):
            assert back({**base, r: M // 2}, attention(**{field: M // 2})) == INVALID, (r, field)


def test_block_norm_overlaps(lib):
    M = 1 << 30
    fields = ("h", "residual", "gate", "scale", "post_weight", "post_bias", "weight", "bias")
    inputs = {n: (20 + i) * M for i, n in enumerate(fields)}
    for gate_rows, gate_bytes in ((0, 10 * 64 * 4), (1, 10 * 4)):
        a = norm(**inputs, gate_rows=gate_rows)
        rows, par = 10 * 64 * 4, 64 * 4
        length = {"h": rows, "residual": rows, "gate": gate_bytes, **{n: par for n in fields[3:]}, "r": rows, "y": rows, "codes": 640, "steps": 20}
        base = {n: (i + 1) * M for i, n in enumerate(("r", "y", "codes", "steps"))}

        def rc(p):
            return lib.pyg_block_norm(ctypes.byref(a), *[at(p[n]) for n in ("r", "y", "codes", "steps")], None)
        for r in base:
            for o, where in {**base, **inputs}.items():
                if o != r:
                    assert rc({**base, r: where + length[o] - 1}) == INVALID, (r, o)
                    assert rc({**base, r: where - length[r] + 1}) == INVALID, (r, o)
        need = size(lib.pyg_block_norm_backward_workspace, ctypes.byref(a))[1]
        grads = ["grad_" + n for n in fields]
        names = ["grad_r", "grad_y", *grads, "ws"]
        base = {n: (i + 1) * M for i, n in enumerate(names)}
        length = {**length, "grad_r": rows, "grad_y": rows, "ws": need, **{"grad_" + n: length[n] for n in fields}}

        def back(p):
            return lib.pyg_block_norm_backward(ctypes.byref(a), *[at(p[n]) for n in names], need, None)
        for r in (*grads, "ws"):
            for o, where in {**base, **inputs}.items():
                if o != r:
                    assert back({**base, r: where + length[o] - 1}) == INVALID, (r, o)
                    assert back({**base, r: where - length[r] + 1}) == INVALID, (r, o)


def test_checkpoint_and_dense_overlaps(lib):
    M = 1 << 30
    for dtype, e in ((0, 4), (1, 2)):
        length = dict(x=10 * 100 * e, codes=10 * 128, steps=10 * 4)
        base = {n: (i + 1) * M for i, n in enumerate(length)}
        for r, o in (("codes", "x"), ("steps", "x"), ("steps", "codes"), ("codes", "steps")):
            for where in (base[o] + length[o] - 1, base[o] - length[r] + 16):  # codes lie on 16 bytes
                p = {**base, r: where // 16 * 16}
                assert lib.pyg_activation_checkpoint(at(p["x"]), dtype, 10, 100, at(p["codes"]), at(p["steps"]), None) == INVALID, (r, o)
                if o == "x":
                    assert lib.pyg_checkpoint_restore(at(p["codes"]), at(p["steps"]), 10, 100, at(p["x"]), dtype, None) == INVALID, (r, o)
        need = size(lib.pyg_dense_transform_backward_workspace, dtype, 1000, 64, 32)[1]
        length = dict(g=1000 * 32 * e, theta=64 * 32 * e, codes=1000 * 64, steps=1000 * 2, gx=1000 * 64 * e, gt=64 * 32 * e, ws=need)
        base = {n: (i + 1) * M for i, n in enumerate(length)}

        def rc(p):
            return lib.pyg_dense_transform_backward(at(p["g"]), dtype, 1000, 32, at(p["theta"]), 64, at(p["codes"]), at(p["steps"]),
                                                    at(p["gx"]), at(p["gt"]), at(p["ws"]), need, None)
        for r in ("gx", "gt", "ws"):
            for o in base:
                if o != r:
                    assert rc({**base, r: base[o] + length[o] - 1}) == INVALID, (r, o)
                    assert rc({**base, r: base[o] - length[r] + 1}) == INVALID, (r, o)


def test_attention_backward_workspace_is_what_is_used(lib):
    """The workspace holds delta, the table's share of every workgroup (32 rows where wavefronts work alone, 128
    elsewhere, times the key ranges) and the shares of the one split that the call takes."""
    def need(**change):
        a = attention(**change)
        status, n = size(lib.pyg_global_attention_backward_workspace, ctypes.byref(a))
        assert status == PYG_OK
        return n, a

    def total(*parts):
        return sum(-(-n // 256) * 256 for n in parts)
    # four wavefronts a workgroup, no heads shared
    n, a = need(B=1, Nq=9000, Nk=9000, H=16, Hkv=16)
    assert n == total(9000 * 16 * 4, (9000 // 128 + 2) * 16 * 8 * 4)
    n, _ = need(B=1, Nq=9000, Nk=9000, H=16, Hkv=16, table=None)
    assert n == total(9000 * 16 * 4)
    # and shared by four: the key tiles' 71 * 4 workgroups times the 4 heads of each
    n, _ = need(B=1, Nq=9000, Nk=9000, H=16, Hkv=4)
    assert n == total(9000 * 16 * 4, (9000 // 128 + 2) * 16 * 8 * 4, 2 * 4 * 9000 * 4 * 32 * 4)
    # lone wavefronts: no shares of heads
    n, _ = need(B=100, Nq=3000, Nk=3000, H=16, Hkv=4)
    assert n == total(3000 * 16 * 4, (3000 // 32 + 101) * 16 * 8 * 4)
    # few queries over a long history, also where there are more than 1,024: ranges of keys for dQ
    for nq, heads, ranges in ((1, 8, 128), (2000, 2, 8)):
        n, _ = need(B=1, Nq=nq, Nk=100_000, H=heads, Hkv=heads)
        assert n == total(nq * heads * 4, (nq // 32 + 2) * ranges * heads * 8 * 4, ranges * nq * heads * 32 * 4)


def test_gradients_that_are_not_wanted(lib):
    """Neither arrays nor workspace for them."""
    def need(**change):
        status, n = size(lib.pyg_global_attention_backward_workspace, ctypes.byref(attention(B=1, Nq=9000, Nk=9000, H=16, Hkv=4, **change)))
        assert status == PYG_OK
        return n
    delta = 9000 * 16 * 4
    assert need(skip=4) == need() - (9000 // 128 + 2) * 16 * 8 * 4 and need(skip=2) == need() - 2 * 4 * 9000 * 4 * 32 * 4
    assert need(skip=7) == need(skip=6) == delta
    a = attention(B=1, Nq=1, Nk=100_000, H=8, Hkv=8)
    b = attention(B=1, Nq=1, Nk=100_000, H=8, Hkv=8, skip=5)
    assert size(lib.pyg_global_attention_backward_workspace, ctypes.byref(b))[1] == 256 < size(lib.pyg_global_attention_backward_workspace, ctypes.byref(a))[1]

    def back(a, gq=D_, gk=B_, gv=C_, gt=A, ws=at(5 << 30)):
        return lib.pyg_global_attention_backward(ctypes.byref(a), at(6 << 30), at(7 << 30), at(8 << 30), at(9 << 30), at(10 << 30),
                                                 at(11 << 30), None, gq, gk, gv, gt, ws, 1 << 30, None)
    assert back(attention(skip=7), None, None, None, None) == PYG_OK  # nothing to do
    assert back(attention(skip=1), gk=None) == INVALID and back(attention(skip=2), gq=None) == INVALID
    # the dense transform's: N = 0 leaves nothing to launch
    dense = lib.pyg_dense_transform_backward
    assert dense(None, 0, 0, 32, B_, 64, None, None, D_, None, None, 0, None) == PYG_OK
    assert dense(None, 0, 0, 32, B_, 64, None, None, D_, A, None, 0, None) == WORKSPACE


def test_dense_sizes_are_refused_before_anything_is_launched(lib):
    """A grid that one of the two results cannot have, also where the other could be made first."""
    def rc(N, Fi, Fo, gx, gt):
        return lib.pyg_dense_transform_backward(A, 0, N, Fo, B_, Fi, C_, C_, gx, gt, D_, 1 << 62, None)
    assert rc(1, 1 << 23, 1 << 23, D_, A) == UNSUPPORTED and rc(1, 1 << 23, 1 << 23, None, A) == UNSUPPORTED
    assert rc((1 << 31) - 1, 1 << 23, 1, D_, None) == UNSUPPORTED


def test_block_norm_codes_lie_on_16_bytes(lib):
    """As the other calls that read and write them want it."""
    a = norm()
    assert lib.pyg_block_norm(ctypes.byref(a), at(1 << 30), at(2 << 30), at((3 << 30) + 8), at(4 << 30), None) == INVALID
