"""Chunks of new tokens on a compressed cache in 64 bits: Algorithm 1 token by token from given
slots, the attention of every token, and bounds on what the kernels' arithmetic may be off by."""
from __future__ import annotations

import numpy as np

from tests.packed_reference import HALF


class Unit:
    """One kv head of one row: closed slots and the open one, its z, and mean absolute values (the
    scale of the rounding of its sums)."""

    def __init__(self, K, V, z):
        self.K, self.V = [np.array(x) for x in K], [np.array(x) for x in V]
        self.AK, self.AV = [np.abs(x) for x in K], [np.abs(x) for x in V]
        self.fresh = [False] * len(self.K)   # states formed by this chunk (rounded), not stored slots
        self.z, self.tokens = float(z), 0

    def update(self, k, v, omega, alpha):
        k = k.copy()
        k[0] = 0.0
        self.tokens += 1
        if alpha and self.K:
            z, zn = self.z, self.z + omega
            for S, A, x in ((self.K, self.AK, k), (self.V, self.AV, v)):
                S[-1] = (S[-1] * z + x * omega) / zn
                A[-1] = (A[-1] * z + np.abs(x) * omega) / zn
            self.z, self.fresh[-1] = zn, True
        else:
            for S, A, x in ((self.K, self.AK, k), (self.V, self.AV, v)):
                S.append(x.copy())
                A.append(np.abs(x))
            self.z = omega
            self.fresh.append(True)
        return len(self.K) - 1

    def state_error(self, u):
        """Rounding of a state formed by the chunk: to the type, plus its fp32 sums and omegas."""
        return u, (self.tokens + 8) * 2.0 ** -24 + 2.0 ** -20

    def attend(self, q, u):
        """Output of one query (element 0 unused) and its bound."""
        q = q.copy()
        q[0] = 0.0
        d = len(q)
        K, V, AV = np.stack(self.K), np.stack(self.V), np.stack(self.AV)
        fresh = np.array(self.fresh)[:, None]
        r, f = self.state_error(u)
        eK = np.where(fresh, r * np.abs(K) + f * np.stack(self.AK), 0.0)
        eV = np.where(fresh, r * np.abs(V) + f * AV, 0.0)
        s = K @ q / np.sqrt(d)
        es = (eK @ np.abs(q) + (d + 8) * 2.0 ** -24 * (np.abs(K) @ np.abs(q))) / np.sqrt(d)
        p = np.exp(s - s.max())
        p /= p.sum()
        o = p @ V
        g = (len(s) + 32) * 2.0 ** -24
        pe = p * (u + g + 2 * es)   # a probability: rounded to the type, its score
        bound = u * np.abs(o) + pe @ np.abs(V) + pe.sum() * np.abs(o) + p @ eV
        return o, 1.15 * bound + 1e-30


class Reference:
    """Units of a layer from slots K, V [B, Hkv, S, d], lengths, z (float64 numpy of the stored
    values); chunks as packed arrays."""

    def __init__(self, K, V, lengths, z, hq, bias=0.0, omega="lead", shared=False, dtype="bf16"):
        self.B, self.hkv = lengths.shape
        self.G = hq // self.hkv
        self.bias, self.omega, self.shared, self.u = bias, omega, shared, HALF[dtype]
        self.units = [[Unit(K[b, g, :lengths[b, g]], V[b, g, :lengths[b, g]], z[b, g])
                       for g in range(self.hkv)] for b in range(self.B)]

    def _omega(self, q, g):
        if self.omega == "uniform":
            return 1.0
        w = np.maximum(1 / (1 + np.exp(-q[g * self.G:(g + 1) * self.G, 0])), 2.0 ** -100)
        return float(w[0] if self.omega == "lead" else w.mean())

    def chunk(self, q, k, v, lens, commit=None, attend=True):
        """(out, bound [T, Hq, d], slot [T, Hkv]) of a chunk; afterwards the units hold row b's first
        commit[b] tokens (default: none)."""
        import copy
        T, hq, d = q.shape
        out, bound = np.zeros((T, hq, d)), np.zeros((T, hq, d))
        slot = np.full((T, self.hkv), -1)
        lo = 0
        for b, n in enumerate(lens):
            keep = 0 if commit is None else commit[b]
            for g in range(self.hkv):
                unit = copy.deepcopy(self.units[b][g])
                dg = 0 if self.shared else g
                for t in range(lo, lo + n):
                    if t - lo == keep:
                        kept = copy.deepcopy(unit)
                    s = unit.update(k[t, g], v[t, g], self._omega(q[t], dg), k[t, dg, 0] > self.bias)
                    if t - lo < keep:
                        slot[t, g] = s
                    if attend:
                        for h in range(g * self.G, (g + 1) * self.G):
                            out[t, h], bound[t, h] = unit.attend(q[t, h], self.u)
                self.units[b][g] = kept if keep < n else unit
            lo += n
        return out, bound, slot

    def lengths(self):
        return np.array([[len(u.K) for u in row] for row in self.units])

    def check_cache(self, cache, layer=0):
        """The cache holds these units: lengths exact, slots and z within their rounding."""
        L = self.lengths()
        assert (cache.lengths(layer).cpu().numpy() == L).all(), "lengths"
        dense = max(1, int(L.max()))
        K, V, z = (x.float().cpu().numpy().astype(np.float64) for x in cache.export(layer, dense))
        for b, row in enumerate(self.units):
            for g, u in enumerate(row):
                r, f = u.state_error(self.u)
                n = len(u.K)
                for got, S, A, what in ((K[b, g], u.K, u.AK, "keys"), (V[b, g], u.V, u.AV, "values")):
                    assert (got[n:] == 0).all()
                    if n == 0:
                        continue
                    S, A = np.stack(S), np.stack(A)
                    fresh = np.array(u.fresh)[:, None]
                    tol = np.where(fresh, 1.1 * (r * np.abs(S) + f * A), 0.0)
                    err = np.abs(got[:n] - S)
                    assert (err <= tol).all(), f"{what} of unit {b},{g}: {np.max(err - tol):.3e} over"
                if n:
                    assert abs(z[b, g] - u.z) <= u.z * 2 * f, f"z of unit {b},{g}: {z[b, g]} for {u.z}"

    def restart(self, cache, layer=0):
        """Take the cache's stored slots as they are (a later chunk starts from rounded ones)."""
        L = cache.lengths(layer).cpu().numpy()
        K, V, z = (x.float().cpu().numpy().astype(np.float64) for x in cache.export(layer, max(1, int(L.max()))))
        self.units = [[Unit(K[b, g, :L[b, g]], V[b, g, :L[b, g]], z[b, g]) for g in range(self.hkv)]
                      for b in range(self.B)]
