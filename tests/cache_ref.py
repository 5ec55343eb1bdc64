"""The receiver's side written out plainly in 64 bits (numpy): rotary positions,
four-bit groups, the page layout, page bookkeeping and attention.  Shares no
code with the HIP path."""
from __future__ import annotations

import math

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def to_f64(t):
    """A torch tensor of any float type as a numpy float64 array."""
    return t.detach().cpu().double().numpy()


# ---- rotary ---------------------------------------------------------------


def rotate(x, freq, delta, amplitude=1.0, interleaved=False, transpose=False):
    """x [..., D], delta [...] (whole numbers), freq [R/2] turns per position."""
    R = 2 * len(freq)
    turn = np.asarray(delta, np.float64)[..., None] * np.asarray(freq)
    ang = 2 * np.pi * (turn - np.floor(turn)) * (-1 if transpose else 1)
    c, s = np.cos(ang) * amplitude, np.sin(ang) * amplitude
    y = np.array(x, np.float64)
    i, j = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    a, b = x[..., i].astype(np.float64), x[..., j].astype(np.float64)
    y[..., i] = a * c - b * s
    y[..., j] = b * c + a * s
    return y


def pair_size(x, R, interleaved):
    """|x| + |y| of the pair that each value belongs to (0 behind the rotated ones)."""
    out = np.zeros(x.shape)
    i, j = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    out[..., i] = out[..., j] = np.abs(x[..., i]) + np.abs(x[..., j])
    return out


# ---- four bits --------------------------------------------------------------


def quantise(x):
    """(codes [..., D], scale bytes [..., D/32]) of rows x [..., D] in float64."""
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, 32)
    bad = ~np.isfinite(g).all(-1)
    top = np.where(bad, 0.0, np.abs(np.where(np.isfinite(g), g, 0.0)).max(-1))
    e = np.full(top.shape, -124, int)
    for k in range(-124, 126):          # the least with top <= 7 * 2^e
        e = np.where((e == k) & (top > 7.0 * 2.0 ** k) & (k < 125), k + 1, e)
    z = np.where(np.isfinite(g), np.abs(g), 0.0) / 2.0 ** e[..., None]
    d = np.abs(z[..., None] - LEVELS)
    near = d.min(-1, keepdims=True)
    # the nearest level; of two the one of even number (they are neighbours)
    hit = d == near
    first = hit.argmax(-1)
    two = hit.sum(-1) == 2
    code = np.where(two & (first % 2 == 1), first + 1, first)
    code = code + 8 * np.signbit(g)
    code = np.where(bad[..., None], 0, code)
    return code.reshape(x.shape).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def values(code, scale):
    v = LEVELS[code & 7] * np.where(code & 8, -1.0, 1.0)
    s = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return (v.reshape(*v.shape[:-1], -1, 32) * s[..., None]).reshape(code.shape)


# ---- layout: one unit (page, layer, head) -----------------------------------


def unpack(unit, P, D):
    """Key and value codes [P][D] and scale bytes [P][D/32] of a unit's bytes."""
    n, s, W = P * D // 2, P * D // 32, D // 32
    kb = unit[:n].reshape(P, D // 2)
    vb = np.empty((P, D // 2), np.uint8)
    vs = np.empty((P, W), np.uint8)
    vraw, sraw = unit[n:2 * n], unit[2 * n + s:]
    for t in range(P):
        for r in range(16):
            at = ((t // 4 * 16 + r) * 4 + t % 4) * W
            vb[t, r * W:(r + 1) * W] = vraw[at:at + W]
        for g in range(W):
            vs[t, g] = sraw[(t // 4 * W + g) * 4 + t % 4]
    ks = unit[2 * n:2 * n + s].reshape(P, W)

    def codes(b):
        return np.stack([b & 15, b >> 4], -1).reshape(P, D)

    return codes(kb), ks.copy(), codes(vb), vs


def pack(kc, ks, vc, vs):
    P, D = kc.shape
    W = D // 32

    def pairs(c):
        return c[:, 0::2] | (c[:, 1::2] << 4)

    vb, v = pairs(vc), np.empty((P // 4, 16, 4, W), np.uint8)
    s = np.empty((P // 4, W, 4), np.uint8)
    for t in range(P):
        v[t // 4, :, t % 4] = vb[t].reshape(16, W)
        s[t // 4, :, t % 4] = vs[t]
    return np.concatenate([pairs(kc).ravel(), v.ravel(), ks.ravel(), s.ravel()])


class Model:
    """The cache's state on the host: pool bytes, refs, table, lens."""

    def __init__(self, pool, refs, table, lens, D, P):
        self.pool, self.refs, self.table, self.lens = (np.array(x) for x in (pool, refs, table, lens))
        self.D, self.P = D, P
        self.width = self.table.shape[1]

    def held(self, s):
        return -(-int(self.lens[s]) // self.P)

    def free_pages(self):
        return [int(p) for p in np.flatnonzero(self.refs == 0)]

    def _save(self):
        return self.refs.copy(), self.table.copy(), self.lens.copy()

    def _restore(self, s):
        self.refs, self.table, self.lens = s

    def free(self, seqs):
        for s in seqs:
            if 0 <= s < len(self.lens):
                for j in range(self.held(s)):
                    p = self.table[s, j]
                    self.table[s, j] = -1
                    if 0 <= p < len(self.refs) and self.refs[p] > 0:
                        self.refs[p] -= 1
                self.lens[s] = 0

    def extend(self, seqs, add):
        ok = [0 <= s < len(self.lens) for s in seqs]
        if not all(ok) or len(set(seqs)) < len(seqs) or any(a < 0 for a in add) or any(
                self.lens[s] + a > self.width * self.P for s, a in zip(seqs, add)):
            return -1
        need = [-(-(int(self.lens[s]) + a) // self.P) - self.held(s) for s, a in zip(seqs, add)]
        free = self.free_pages()
        if sum(need) > len(free):
            return sum(need) - len(free)
        for s, a, k in zip(seqs, add, need):
            h = self.held(s)
            for j in range(k):
                p = free.pop(0)
                self.table[s, h + j] = p
                self.refs[p] = 1
            self.lens[s] += a
        return 0

    def fork(self, parents, children, copy):
        n = len(self.lens)
        if any(not 0 <= s < n for s in [*parents, *children]) or len(set(children)) < len(children) \
                or set(parents) & set(children):
            return -1
        before = self._save()
        self.free(children)
        free, pool = self.free_pages(), self.pool
        need = sum(self.held(p) if copy else int(self.lens[p] % self.P != 0) for p in parents)
        if need > len(free):
            self._restore(before)
            return need - len(free)
        for p, c in zip(parents, children):
            for j in range(self.held(p)):
                page = int(self.table[p, j])
                if copy or (j == self.held(p) - 1 and self.lens[p] % self.P):
                    new = free.pop(0)
                    pool[new] = pool[page]
                    self.refs[new] = 1
                    page = new
                else:
                    self.refs[page] += 1
                self.table[c, j] = page
            self.lens[c] = self.lens[p]
        return 0

    def compact(self, src, dst, idx, counts):
        """idx(i, l, h): the list of entry i, layer l, head h."""
        n, keep = len(self.lens), len(idx(0, 0, 0)) if src else 0
        counts = [keep] * len(src) if counts is None else counts
        if any(not 0 <= s < n for s in [*src, *dst]) or len(set(dst)) < len(dst) or any(
                not 0 <= k <= keep for k in counts) or any(
                s in dst and d != s for s, d in zip(src, dst)):
            return -1
        before, pool = self._save(), self.pool.copy()
        rows = [(int(self.lens[s]), self.table[s].copy()) for s in src]
        self.free([d for s, d in zip(src, dst) if s != d])
        free = self.free_pages()
        need = sum(-(-k // self.P) for k in counts)
        if need > len(free):
            self._restore(before)
            return need - len(free)
        self.free([d for s, d in zip(src, dst) if s == d])
        D, P = self.D, self.P
        units = {}

        def unit(page, l, h):
            if (page, l, h) not in units:
                units[page, l, h] = unpack(pool[page, l, h], P, D)
            return units[page, l, h]

        for i, d in enumerate(dst):
            for j in range(-(-counts[i] // P)):
                new = free.pop(0)
                self.table[d, j] = new
                self.refs[new] = 1
                for l in range(pool.shape[1]):
                    for h in range(pool.shape[2]):
                        kc, vc = np.zeros((P, D), np.uint8), np.zeros((P, D), np.uint8)
                        ks, vs = np.full((P, D // 32), 3, np.uint8), np.full((P, D // 32), 3, np.uint8)
                        for t in range(min(P, counts[i] - j * P)):
                            s = int(idx(i, l, h)[j * P + t])
                            if 0 <= s < rows[i][0]:
                                u = unit(int(rows[i][1][s // P]), l, h)
                                kc[t], ks[t], vc[t], vs[t] = (x[s % P] for x in u)
                        self.pool[new, l, h] = pack(kc, ks, vc, vs)
            self.lens[d] = counts[i]
        return 0

    def read(self, s, l, h, n=None):
        """Keys and values [len][D] of a sequence in one layer and head (NaN groups as NaN; a hole in
        the table as None in the list of held positions)."""
        n = int(self.lens[s]) if n is None else n
        k, v, there = np.zeros((n, self.D)), np.zeros((n, self.D)), np.zeros(n, bool)
        for j in range(-(-n // self.P)):
            p = int(self.table[s, j])
            if not 0 <= p < len(self.refs):
                continue
            kc, ks, vc, vs = unpack(self.pool[p, l, h], self.P, self.D)
            a, b = j * self.P, min(n, (j + 1) * self.P)
            k[a:b], v[a:b] = values(kc, ks)[:b - a], values(vc, vs)[:b - a]
            there[a:b] = True
        return k, v, there


# ---- attention --------------------------------------------------------------


def attend(q, k, v, limit, there, scale):
    """One query row over keys and values [T][D]: (out [D], lse, bound on the logits' error in units
    of 2^-24, sum p|v| and 2^-126 sum |v|: what weights below fp32's normal range come to).  Positions from `limit` on and those not `there` count for nothing."""
    T, D = k.shape
    see = there & (np.arange(T) < limit)
    if not see.any():
        return np.zeros(D), -math.inf, 0.0, np.zeros(D), 0.0
    kk, vv = k[see], v[see]
    x = scale * (kk @ q)
    if np.isnan(x).any():
        return np.full(D, np.nan), math.nan, 0.0, np.zeros(D), 0.0
    top = x.max()
    w = np.exp(x - top)
    z = w.sum()
    p = w / z
    # a sum of D products in fp32, and the rounding of the scaled logit
    err = ((D + 4) * scale * (np.abs(kk) @ np.abs(q)) + 2 * np.abs(x)).max()
    return p @ vv, top + math.log(z), err, p @ np.abs(vv), 2.0 ** -126 * np.abs(vv).sum(0)
