"""Attention over the graphs of a batch in 64 bits, and how far a correct
implementation in fp32 (or with bf16 operands) may be from it, value by value."""
import math

import torch

U32 = 2.0 ** -24  # half a step of fp32, relative


def lengths(kind, rng, B, most):
    if kind == "one":
        return [1] * B
    return [int(n) for n in rng.integers(0, most + 1, B)]


def attention(q, k, v, qn, kn, table=None, lut=None, causal=False, scale=None, grad=None):
    """out (and with `grad` the gradients) with bounds: {name: (value, bound)}. CPU tensors; bf16 ones are
    rounded at P, dS and every result, as the kernels say they do."""
    dt = q.dtype
    half = torch.finfo(dt).eps / 2 if dt != torch.float32 else 0.0
    H, D = q.shape[1:]
    Hkv = k.shape[1]
    G = H // Hkv
    c = D ** -0.5 if scale is None else scale
    Q, K, V = (t.double() for t in (q, k, v))
    names = ["out"] + (["grad_q", "grad_k", "grad_v"] if grad is not None else [])
    val = {n: torch.zeros(t.shape, dtype=torch.float64) for n, t in zip(names, (q, q, k, v))}
    bnd = {n: torch.zeros(t.shape, dtype=torch.float64) for n, t in zip(names, (q, q, k, v))}
    if grad is not None and table is not None:
        names.append("grad_table")
        val["grad_table"], bnd["grad_table"] = (torch.zeros(table.shape, dtype=torch.float64) for _ in range(2))
    q0 = k0 = 0
    R = (len(lut) - 1) // 2 if lut is not None else 0
    for n, m in zip(qn, kn):
        off = torch.arange(m)[None] - torch.arange(m - n, m)[:, None]
        idx = lut.long()[off.clamp(-R, R) + R] if lut is not None else None
        for h in range(H):
            hk = h // G
            x, y, z = Q[q0:q0 + n, h], K[k0:k0 + m, hk], V[k0:k0 + m, hk]
            prod, pmag = (x @ y.T) * c, (x.abs() @ y.abs().T) * c
            bias = table.double()[idx, h] if table is not None else torch.zeros(n, m, dtype=torch.float64)
            a = prod + bias
            if causal:
                a = torch.where(off <= 0, a, -math.inf)
            top = a.max(1, keepdim=True).values if m else torch.zeros(n, 1, dtype=torch.float64)
            seen = torch.isfinite(top) if m else torch.zeros(n, 1, dtype=torch.bool)
            e = torch.where(seen, torch.exp(a - torch.where(seen, top, 0.0)), 0.0)
            tot = e.sum(1, keepdim=True)
            p = torch.where(seen, e / torch.where(tot > 0, tot, 1.0), 0.0)
            fin = torch.where(torch.isfinite(bias), bias.abs(), 0.0)
            # a's error: D products summed in any order, the bias over c rounded, s, c2 s and the exponent's rounding;
            # where a lowest bias swallows the product both do
            aerr = torch.where(fin < 1e30, ((D + 4) * pmag + 4 * (fin + pmag) + 4 * torch.where(seen, top.abs(), 0.0)) * U32, 0.0)
            worst = aerr.max(1, keepdim=True).values if m else torch.zeros(n, 1, dtype=torch.float64)
            prel = 2 * worst + (m + 12) * U32  # of p: the exponent, exp2, the sum and the division
            o, omag = p @ z, p @ z.abs()
            oerr = (prel + m * U32 + half) * omag
            val["out"][q0:q0 + n, h] = o
            bnd["out"][q0:q0 + n, h] = oerr + (half + U32) * (o.abs() + oerr)
            if grad is None:
                continue
            g = grad[q0:q0 + n, h].double()
            dp, dmag = g @ z.T, g.abs() @ z.abs().T
            delta = (g * o).sum(1, keepdim=True)
            derr = (g.abs() * bnd["out"][q0:q0 + n, h]).sum(1, keepdim=True) + (D + 2) * U32 * (g.abs() * o.abs()).sum(1, keepdim=True)
            ds = p * (dp - delta)
            dserr = p * ((prel + 2 * U32) * (dp - delta).abs() + (D + 2) * U32 * dmag + derr)
            dsr = dserr + half * (ds.abs() + dserr)  # rounded for the matrix cores
            sl_q, sl_k = slice(q0, q0 + n), slice(k0, k0 + m)
            val["grad_q"][sl_q, h] = c * ds @ y
            bnd["grad_q"][sl_q, h] = c * (dsr + (m + 2) * U32 * ds.abs()) @ y.abs()
            val["grad_k"][sl_k, hk] += c * ds.T @ x
            bnd["grad_k"][sl_k, hk] += c * (dsr + (n * G + 2) * U32 * ds.abs()).T @ x.abs()
            val["grad_v"][sl_k, hk] += p.T @ g
            bnd["grad_v"][sl_k, hk] += ((prel + half + (n * G + 2) * U32) * p).T @ g.abs()
            if "grad_table" in val:
                for t, w in (("val", ds), ("bnd", dserr + (n + m + 64) * U32 * ds.abs())):
                    (val if t == "val" else bnd)["grad_table"][:, h] += torch.bincount(idx.reshape(-1), w.reshape(-1), len(table))
        q0, k0 = q0 + n, k0 + m
    for name in names[1:]:
        bnd[name] = bnd[name] + (half + U32) * (val[name].abs() + bnd[name])
    return {n: (val[n], bnd[n] + 1e-30) for n in names}


def close(got, ref, what):
    for name, t in got.items():
        val, bound = ref[name]
        t = t.detach().cpu().double()
        assert t.shape == val.shape, f"{what} {name}: shape"
        err = (t - val).abs()
        bad = ~(err <= bound)
        assert not bad.any(), (f"{what} {name}: {int(bad.sum())} of {bad.numel()} values off, worst error over bound "
                               f"{float((err / bound).max()):.3g}, first at {bad.nonzero()[0].tolist()}")
