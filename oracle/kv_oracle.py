"""Plain model of the paged 4-bit KV cache: numpy, one token at a time, 64-bit attention.

Written from the definitions in mars_kv.h, without any code of the library.  Number formats are
tables; conversions search them.  The quotients of the quantiser are fp32 by definition, so codes
and scales can be compared bit for bit; everything else is evaluated in 64 bits.
"""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E4M3 = np.array([m * 2.0 ** -9 for m in range(8)]
                + [(1 + m / 8) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)][:-1])   # 0 .. 448

OK, BAD_TREE, NO_ROOM, OUT_OF_PAGES, BAD_PATH, BAD_FORK = 0, 1, 5, 7, 8, 9


def nearest(x, table):
    """Index of the nearest entry of an ascending table, ties to the even index, saturating."""
    x = np.minimum(np.asarray(x, np.float64), table[-1])
    hi = np.clip(np.searchsorted(table, x), 1, len(table) - 1)
    lo = hi - 1
    up, down = table[hi] - x, x - table[lo]
    return np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))


def quantise(x, g):
    """Codes 0..15 [..., d] and scale bytes [..., d/16] of rows x; g broadcasts over [..., d/16]."""
    x = np.where(np.isnan(x), 0.0, np.asarray(x, np.float64)).astype(np.float32)
    y = x.reshape(*x.shape[:-1], -1, 16)
    g = np.broadcast_to(np.asarray(g, np.float32), y.shape[:-1])
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        a = np.abs(y).max(-1)
        s = nearest(a / np.float32(6) / g, E4M3)
        sg = E4M3[s].astype(np.float32) * g
        t = np.where(sg[..., None] > 0, y / sg[..., None], np.float32(0))
    c = nearest(np.abs(t), E2M1) | np.where(np.signbit(t), 8, 0)
    return c.reshape(x.shape).astype(np.uint8), s.astype(np.uint8)


def values(c, s, g):
    """64-bit values of codes [..., d] with scale bytes [..., d/16] (any byte of the format)."""
    mag = E2M1[c & 7] * np.where(c & 8, -1.0, 1.0)
    sc = np.where((s & 0x7f) == 0x7f, np.nan, np.append(E4M3, 0.0)[s & 0x7f]) * np.where(s & 0x80, -1.0, 1.0)
    return mag * np.repeat(sc, 16, -1) * g


class Model:
    """Tables and rows of one cache; rows are kept per (page, slot) as codes and scales."""

    def __init__(self, layers, num_pages, kv_heads, d, page, seqs, width, scales):
        self.L, self.P, self.H, self.d, self.page, self.S, self.W = layers, num_pages, kv_heads, d, page, seqs, width
        self.scales = np.asarray(scales, np.float32)
        self.code = np.zeros((layers, num_pages, page, kv_heads, 2, d), np.uint8)
        self.scale = np.zeros((layers, num_pages, page, kv_heads, 2, d // 16), np.uint8)
        self.table = np.full((seqs, width), -1, np.int32)
        self.len = np.zeros(seqs, np.int32)
        self.held = np.zeros(seqs, np.int32)
        self.refs = np.zeros(num_pages, np.int32)

    def cap(self, b):
        return self.held[b] * self.page

    def at(self, b, pos):
        return self.table[b, pos // self.page], pos % self.page

    def free_pages(self):
        return np.flatnonzero(self.refs == 0)

    def free_bits(self):
        w = np.zeros((self.P + 31) // 32, np.uint32)
        for p in self.free_pages():
            w[p >> 5] |= np.uint32(1 << (p & 31))
        return w.view(np.int32)

    def resize(self, extra):
        status = np.zeros(self.S, np.int32)
        want = self.held.copy()
        for b in range(self.S):
            ex = int(extra[b])
            if ex < -1:
                continue
            w = 0 if ex == -1 else -(-(int(self.len[b]) + ex) // self.page)
            if w > self.W:
                status[b] = NO_ROOM
                continue
            want[b] = w
            for c in range(w, self.held[b]):
                self.refs[self.table[b, c]] -= 1
                self.table[b, c] = -1
            self.held[b] = min(self.held[b], w)
            if ex == -1:
                self.len[b] = 0
        free, short = list(self.free_pages()), False
        for b in range(self.S):
            need = int(want[b] - self.held[b])
            if need <= 0:
                continue
            short = short or need > len(free)
            if short:
                status[b] = OUT_OF_PAGES
                continue
            for c in range(need):
                p = free.pop(0)
                self.table[b, self.held[b] + c] = p
                self.refs[p] = 1
            self.held[b] = want[b]
        return status

    def append(self, layer, k, v, count=None):
        B, N = k.shape[:2]
        status = np.zeros(B, np.int32)
        for b in range(B):
            n = N if count is None else int(np.clip(count[b], 0, N))
            if n and self.len[b] + n > self.cap(b):
                status[b] = NO_ROOM
                continue
            for kv, x in ((0, k), (1, v)):
                if n:
                    c, s = quantise(x[b, :n], self.scales[layer, kv][None, :, None])
                    for i in range(n):
                        p, slot = self.at(b, self.len[b] + i)
                        self.code[layer, p, slot, :, kv] = c[i]
                        self.scale[layer, p, slot, :, kv] = s[i]
        return status

    def rows(self, layer, b, first, n):
        """K, V [n, H, d] in 64 bits."""
        c = np.stack([self.code[layer, p, s] for p, s in (self.at(b, first + i) for i in range(n))])
        sc = np.stack([self.scale[layer, p, s] for p, s in (self.at(b, first + i) for i in range(n))])
        return [values(c[:, :, kv], sc[:, :, kv], self.scales[layer, kv].astype(np.float64)[None, :, None])
                for kv in range(2)]

    def commit(self, path, accept):
        B = len(accept)
        status, new = np.zeros(B, np.int32), self.len[:B].copy()
        for b in range(B):
            a = int(accept[b])
            if a == -1:
                continue
            nodes = list(range(a + 1)) if path is None else [int(x) for x in path[b, :max(a, 0) + 1]]
            if a < 0 or len(nodes) != a + 1 or nodes[0] != 0 or any(y <= x for x, y in zip(nodes, nodes[1:])) \
                    or self.len[b] + nodes[-1] >= self.cap(b):
                status[b] = BAD_PATH
                continue
            for j, m in enumerate(nodes):
                (sp, ss), (dp, ds) = self.at(b, self.len[b] + m), self.at(b, self.len[b] + j)
                self.code[:, dp, ds] = self.code[:, sp, ss]
                self.scale[:, dp, ds] = self.scale[:, sp, ss]
            new[b] += a + 1
        return new, status

    def fork(self, src, dst):
        status = np.zeros(len(src), np.int32)
        len0, held0, table0 = self.len.copy(), self.held.copy(), self.table.copy()
        claimed, free, short = set(), list(self.free_pages()), False
        for i, (s, d) in enumerate(zip(src, dst)):
            ok = 0 <= s < self.S and 0 <= d < self.S and s != d
            if ok:
                pages = -(-int(len0[s]) // self.page)
                ok = held0[d] == 0 and pages <= held0[s] and (0 <= table0[s, :pages]).all() \
                    and (table0[s, :pages] < self.P).all() and d not in claimed
            if not ok:
                status[i] = BAD_FORK
                continue
            claimed.add(d)
            full, tail = divmod(int(len0[s]), self.page)
            if tail:
                short = short or not free
                if short:
                    status[i] = OUT_OF_PAGES
                    continue
                p = free.pop(0)
                self.table[d, full] = p
                self.refs[p] = 1
                self.code[:, p, :tail] = self.code[:, table0[s, full], :tail]
                self.scale[:, p, :tail] = self.scale[:, table0[s, full], :tail]
            self.table[d, :full] = table0[s, :full]
            for p in table0[s, :full]:
                self.refs[p] += 1
            self.len[d], self.held[d] = len0[s], full + (tail > 0)
        return status

    def pool(self):
        """The pool's bytes [L, P, H, page bytes] and a mask of nothing: every slot as the model has it."""
        L, P, H, d, nb = self.L, self.P, self.H, self.d, self.page // 16
        out = np.zeros((L, P, H, nb, 18 * d), np.uint8)
        c = self.code.reshape(L, P, nb, 16, H, 2, d).transpose(0, 1, 4, 2, 5, 3, 6)     # L P H nb 2 16 d
        c = c[..., 0::2] | (c[..., 1::2] << 4)
        out[..., :16 * d] = c.reshape(L, P, H, nb, 16 * d)
        s = self.scale.reshape(L, P, nb, 16, H, 2, d // 16).transpose(0, 1, 4, 2, 5, 3, 6)
        out[..., 16 * d:] = s.reshape(L, P, H, nb, 2 * d)
        return out.reshape(L, P, H, nb * 18 * d)


def ancestors(parent, n):
    """(visible [n, n], live [n], status) of one sequence's first n nodes; parent None: a chain."""
    see, live = np.zeros((n, n), bool), np.zeros(n, bool)
    if parent is None:
        return np.tril(np.ones((n, n), bool)), np.ones(n, bool), OK
    par = [int(x) for x in parent[:n]]
    if par and (par[0] != -1 or any(par[i] >= i or par[i] < -1 for i in range(1, n))):
        see[0, 0] = live[0] = True
        return see, live, BAD_TREE
    for i in range(n):
        j = i
        while j >= 0:
            see[i, j] = True
            live[i] = j == 0
            j = par[j]
    return see, live, OK


def attention(m: Model, layer, q, parent=None, count=None, scale=None):
    """64-bit result, which rows have one, the statuses, and what error bounds need: per output the
    probability-weighted |V| and the plain sum of |V|, per row the largest sum of |q||K| times the scale."""
    B, N, Hq, d = q.shape
    G = Hq // m.H
    scale = d ** -0.5 if scale is None else scale
    out, mag, tot = (np.zeros((B, N, Hq, d)) for _ in range(3))
    amp = np.zeros((B, N, Hq))
    live, status = np.zeros((B, N), bool), np.zeros(B, np.int32)
    for b in range(B):
        n = N if count is None else int(np.clip(count[b], 0, N))
        if n == 0:
            continue
        ln = int(m.len[b])
        if ln < 0 or ln + n > m.cap(b):
            status[b] = NO_ROOM
            continue
        see, lv, status[b] = ancestors(None if parent is None else (parent if parent.ndim == 1 else parent[b]), n)
        live[b, :n] = lv
        k, v = m.rows(layer, b, 0, ln + n)
        for i in np.flatnonzero(lv):
            use = np.concatenate([np.arange(ln), ln + np.flatnonzero(see[i])])
            for h in range(Hq):
                qq, kk, vv = q[b, i, h].astype(np.float64), k[use, h // G], v[use, h // G]
                z = kk @ qq * scale
                p = np.exp(z - z.max())
                p /= p.sum()
                out[b, i, h], mag[b, i, h], tot[b, i, h] = p @ vv, p @ np.abs(vv), np.abs(vv).sum(0)
                amp[b, i, h] = (np.abs(kk) @ np.abs(qq)).max() * scale
    return out, live, status, mag, tot, amp
