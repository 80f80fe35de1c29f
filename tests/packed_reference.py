"""Plain causal attention of packed sequences in 64 bits on the CPU, its gradients, and bounds on
what the kernels' arithmetic may be off by (shared by the tests of packed sequences)."""
from __future__ import annotations

import math

import torch

#: Half a rounding step, relative: of bf16 outputs and operands, and of fp32 arithmetic.
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


def dtype_of(name):
    return torch.float32 if name == "fp32" else torch.bfloat16


def cu_of(lens):
    return torch.tensor([0] + list(torch.tensor(lens).cumsum(0)), dtype=torch.int32)


def causal(q, k, v, lens, dout=None):
    """Outputs out, lse (and dq, dk, dv) of CPU tensors [T, heads, d] in float64, each with the bound
    of its error: a dict name -> (value, bound).

    With u half a rounding step of the tensors' type and f = (n + d + 32) 2^-24 for fp32 chains:
      out    rounding u |o|, and P rounded to the type: u P |v|
      lse    e_S and f
      scores chains of d products: e_S = d 2^-24 |q|.|k| / sqrt(d), relative in P (twice: with lse's)
      D      = dO . o with the rounded o: e_D = sum |dO| bound(o); a sequence's first 128 rows
             sum P dP instead: e_D = (2 e_S + f) sum P (|dP| + |D|)
      dS     = P (dP - D): u |dS| (rounded to the type) + P e_D + e_S |dS|
      dq     = sum dS k: sum e_dS |k| + u |dq|;  dk likewise;  dv = sum P dO: sum u P |dO| + u |dv|
    """
    name = "fp32" if q.dtype == torch.float32 else "bf16"
    u = HALF[name]
    q, k, v = q.double(), k.double(), v.double()
    T, Hq, d = q.shape
    G = Hq // k.shape[1]
    res = {x: (torch.zeros(s, dtype=torch.float64), torch.zeros(s, dtype=torch.float64))
           for x, s in dict(out=q.shape, lse=(T, Hq), dq=q.shape, dk=k.shape, dv=k.shape).items()}
    lo = 0
    for n in lens:
        r = slice(lo, lo + n)
        lo += n
        if n == 0:
            continue
        f = (n + d + 32) * 2.0 ** -24
        low = torch.ones(n, n, dtype=torch.float64).tril()
        for h in range(Hq):
            qh, kh, vh = q[r, h], k[r, h // G], v[r, h // G]
            s = (qh @ kh.T) / math.sqrt(d)
            es = (d + 8) * 2.0 ** -24 * ((qh.abs() @ kh.abs().T) / math.sqrt(d) * low).amax() + f
            s = torch.where(low > 0, s, -math.inf)
            lse = torch.logsumexp(s, 1)
            P = torch.exp(s - lse[:, None])
            o = P @ vh
            pu = u + 2 * es   # relative error of a probability
            bo = 1.1 * (u * o.abs() + (pu + f) * (P @ vh.abs() + o.abs())) + 1e-30
            for x, val, err in (("out", o, bo), ("lse", lse, es + f * (1 + lse.abs()))):
                res[x][0][r, h] = val
                res[x][1][r, h] = err
            if dout is None:
                continue
            do = dout[r, h].double()
            dp = do @ vh.T
            D = (do * o).sum(1, keepdim=True)
            dS = P * (dp - D)
            eD = (do.abs() * (bo + f * o.abs())).sum(1, keepdim=True)
            # (the first 128 rows take D from sum P dP, with unrounded probabilities)
            eD[:128] = ((2 * es + f) * P * (dp.abs() + D.abs())).sum(1, keepdim=True)[:128] + (
                f * do.abs() @ vh.abs().T * P).sum(1, keepdim=True)[:128]
            edp = f * (do.abs() @ vh.abs().T)
            eS = (u + 2 * es + f) * dS.abs() + P * (eD + edp)
            sc = 1 / math.sqrt(d)
            for x, hh, val, err in (("dq", h, dS @ kh * sc, (eS @ kh.abs() + f * dS.abs() @ kh.abs()) * sc),
                                    ("dk", h // G, dS.T @ qh * sc, (eS.T @ qh.abs() + f * dS.abs().T @ qh.abs()) * sc),
                                    ("dv", h // G, P.T @ do, (pu + f) * (P.T @ do.abs()))):
                res[x][0][r, hh] += val
                res[x][1][r, hh] += 1.1 * err + 1e-30
    for x in ("dq", "dk", "dv"):
        res[x] = (res[x][0], res[x][1] + u * res[x][0].abs())
    return res


def check(got, want, what):
    value, bound = want
    err = (got.detach().cpu().double() - value).abs()
    bad = ~(err <= bound)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} outside the bound; worst "
                           f"{float((err / bound.clamp_min(1e-300)).nan_to_num(1e9).max()):.2f} of it, largest error "
                           f"{float(err.nan_to_num(1e9).max()):.3e}")
    return float((err / bound.clamp_min(1e-300)).max()) if err.numel() else 0.0
