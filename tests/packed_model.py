"""A plain fp64 model of a layer whose cache is held in 4 bits, in pages: the oracle's layer with rows rounded as the cache rounds
them, and the rules by which pages are taken, shared, copied and given up.  Python loops over units; nothing of the library's."""
from __future__ import annotations

import numpy as np

from oracle import indexmem_oracle as O

LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
SLOTS = 64


def quantise(x: np.ndarray) -> np.ndarray:
    """Rows [..., 128] as the 4-bit cache holds them: per 32 values the smallest power of two u (>= 2^-126) with |x| <= 6 u, then
    the nearest of u * LEVELS, by distance, of two as near the one whose code is even; NaN where the 32 hold an inf or a NaN."""
    x = np.asarray(x, np.float64)
    y = x.reshape(*x.shape[:-1], 4, 32)
    bad = ~np.isfinite(y).all(-1, keepdims=True)
    y = np.where(bad, 0.0, y)
    a = np.abs(y).max(-1, keepdims=True)
    u = np.full(a.shape, 2.0 ** -126)
    for k in range(-126, 128):
        u = np.where(a > 6 * u, 2.0 ** (k + 1), u)
    d = np.abs(np.abs(y / u)[..., None] - LEVELS)
    d = d + np.where(np.arange(8) % 2 == 1, 1e-12, 0.0)   # (y / u has 8 bits: differences are 2^-9 and more, or 0)
    d = np.where(LEVELS * u[..., None] < 2.0 ** 128, d, np.inf)   # (no bf16 value)
    got = np.sign(y) * LEVELS[d.argmin(-1)] * u
    return np.where(bad, np.nan, got).reshape(x.shape)


class PackedModel(O.OracleLayer):
    """The oracle's layer over such a cache; n_pages: size of the pool."""

    def __init__(self, cfg, params, n_pages: int):
        super().__init__(cfg, params)
        self.T = (cfg.capacity + SLOTS - 1) // SLOTS
        self.table = np.full((cfg.batch, cfg.n_kv_heads, self.T), -1, np.int32)
        self.refs = np.zeros(n_pages, np.int32)
        self.status = 0

    def _take(self, needs):
        """needs: per unit (in order) the page indexes that need a new page.  The free pages of the lowest numbers go to them in order;
        a unit that does not get all of its pages gets none, and its share is not passed on.  Returns {unit: new page ids}."""
        free = np.flatnonzero(self.refs == 0)
        at, got = 0, {}
        for unit, pages in needs:
            if at + len(pages) <= len(free) or not pages:
                got[unit] = [int(free[at + i]) for i in range(len(pages))]
            at += len(pages)
        return got

    def append_kv(self, k_new, v_new, pos_new):
        n_new, needs, fits = k_new.shape[2], [], {}
        for u in self.units():
            n = int(self.len[u])
            fits[u] = n + n_new <= self.cfg.capacity
            pages = range(n // SLOTS, (n + n_new - 1) // SLOTS + 1) if fits[u] else []
            needs.append((u, [p for p in pages if self.table[u][p] < 0 or self.refs[self.table[u][p]] > 1]))
            self.status |= 0 if fits[u] else 1
        got = self._take(needs)
        released = []
        for u, pages in needs:
            if u not in got:
                self.status |= 16
            if u not in got or not fits[u]:
                continue
            for p, new in zip(pages, got[u]):
                if self.table[u][p] >= 0:
                    released.append(self.table[u][p])
                self.table[u][p] = new
                self.refs[new] = 1
            n = int(self.len[u])
            k, v = k_new[u], v_new[u]
            self.K[u][n:n + n_new], self.V[u][n:n + n_new] = quantise(k), quantise(v)
            self.Kidx[u][n:n + n_new] = O.key_feature(k, self.p.Uk, self.p.norm_k_w, self.cfg.rms_eps)
            self.pos[u][n:n + n_new] = pos_new[u[0]]
            self.len[u] = self.n_projected[u] = n + n_new
        for page in released:
            self.refs[page] -= 1

    def compact_kv(self, keep, evict):
        needs = []
        for u in self.units():
            k, e = keep[u[0]][u[1]], evict[u[0]][u[1]]
            holes = {int(s) // SLOTS for s in e if s < len(k)}
            needs.append((u, sorted(p for p in holes if self.refs[self.table[u][p]] > 1)))
        got = self._take(needs)
        released = []
        for u, pages in needs:
            if u not in got:
                self.status |= 16
                continue
            k, e = keep[u[0]][u[1]], evict[u[0]][u[1]]
            for src, dst in O.compaction_moves(k, e):
                for a in (self.K, self.V, self.Kidx, self.pos):
                    a[u][dst] = a[u][src]
            for p, new in zip(pages, got[u]):
                released.append(self.table[u][p])
                self.table[u][p] = new
                self.refs[new] = 1
            for p in range(self.T):
                if p * SLOTS >= len(k) and self.table[u][p] >= 0:
                    released.append(self.table[u][p])
                    self.table[u][p] = -1
            self.len[u] = self.n_projected[u] = len(k)
        for page in released:
            self.refs[page] -= 1

    def fork(self, src_of):
        for b, a in enumerate(src_of):
            if a == b:
                continue
            if a < -1 or a >= self.cfg.batch or (a >= 0 and src_of[a] != a):
                self.status |= 32
                continue
            for h in range(self.cfg.n_kv_heads):
                for page in self.table[b, h]:
                    if page >= 0:
                        self.refs[page] -= 1
                if a < 0:
                    self.table[b, h], self.len[b, h], self.n_projected[b, h], self.M[b, h], self.b[b, h] = -1, 0, 0, 0, 0
                    continue
                for page in self.table[a, h]:
                    if page >= 0:
                        self.refs[page] += 1
                n = int(self.len[a, h])
                for x in (self.K, self.V, self.Kidx, self.pos):
                    x[b, h, :n] = x[a, h, :n]
                for x in (self.table, self.len, self.n_projected, self.M, self.b):
                    x[b, h] = x[a, h]

    def attend(self, q, q_pos=None):
        """q [B, n_q, H, D] -> (out, readout, tolerance of out, tolerance of readout), fp64, unrounded."""
        cfg, p = self.cfg, self.p
        B, n_q, H, D = q.shape
        g = H // cfg.n_kv_heads
        out, res, t_out, t_res = (np.zeros(q.shape) for _ in range(4))
        for bi, hi in self.units():
            n = int(self.len[bi, hi])
            K, V = self.K[bi, hi, :n], self.V[bi, hi, :n]
            for s in range(n_q):
                seen = np.ones(n, bool) if q_pos is None else self.pos[bi, hi, :n] <= q_pos[bi, s]
                x = q[bi, s, hi * g:(hi + 1) * g]
                o = O.attend(x, K[seen], V[seen], cfg.softmax_scale)
                m = O.memory_read(x, self.M[bi, hi], self.b[bi, hi], p.Wtheta, cfg.mem_eps)
                gate = O.read_gate(x, p.wg, p.cg)[:, None]
                phi = x @ p.Wtheta.T
                size = gate * (np.abs(phi) @ np.abs(self.M[bi, hi])) / ((phi * phi) @ self.b[bi, hi] + cfg.mem_eps)[:, None]
                out[bi, s, hi * g:(hi + 1) * g], res[bi, s, hi * g:(hi + 1) * g] = o + gate * m, gate * m
                # a weight exp(l - max) / sum is off by the error of its logit: fp32 sums of exact products (2^-24 of the sum of
                # |q k| scale, a few times: below 2^-18 of it) and by fp32 exp and sums (2^-20).  Up to 16 rows a unit it goes into its
                # product as two bf16 parts (2^-17), above as fp16: half a step of 2^-11, and of 2^-31 where it is below 2^-21.  The
                # weights sum to 1, so the output is off by that times the largest |v|.  Memory: 2^-15 of the sum of its terms (phi and M
                # in two bf16 parts each, 2^-16; fp32 sums).  The output's rounding: half a step, 2^-9 to 2^-8 of it.
                big = np.abs(V[seen]).max() if seen.any() and np.isfinite(V[seen]).any() else 0.0
                logit = (np.abs(x) @ np.abs(K[seen]).T).max(initial=0.0) * cfg.softmax_scale if seen.any() else 0.0
                part = 2.0 ** -16 if n_q * g <= 16 else 2.0 ** -12 + 2.0 ** -16
                t = (part + 2.0 ** -18 * 2 * logit) * 2 * big
                t_res[bi, s, hi * g:(hi + 1) * g] = 2.0 ** -15 * size
                t_out[bi, s, hi * g:(hi + 1) * g] = t + 2.0 ** -15 * size
        return out, res, t_out + 2.0 ** -8 * np.abs(out), t_res


def close(got, want, tol):
    """Largest |got - want| / tol, NaN where both are; fails where it is above 1."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape
    assert (np.isnan(got) == np.isnan(want)).all(), "NaN in other places"
    ok = ~np.isnan(want)
    d = np.abs(got - want)[ok] / np.maximum(np.broadcast_to(tol, want.shape)[ok], 1e-37)
    worst = float(d.max(initial=0.0))
    assert worst <= 1.0, f"{worst:.3g} of the tolerance"
    return worst
