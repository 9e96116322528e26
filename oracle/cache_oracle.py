"""Independent CPU model of what runs around a verification call: rotary positions, the paged cache's bookkeeping and the
attention of a drafted block, in float64 numpy from their definitions.  Shares no code with the library."""
from __future__ import annotations

import numpy as np

OK, PAGES, BAD_INDEX = 0, 8, 9


def rope(x, positions, inv_freq, layout, amplitude=1.0, inverse=False):
    """x [..., heads, D], positions [...]: pairs turned by position x frequency, as complex numbers."""
    x = np.asarray(x, dtype=np.float64)
    f = np.asarray(inv_freq, dtype=np.float32).astype(np.float64)
    n = f.size
    turn = np.exp((-1j if inverse else 1j) * np.asarray(positions, dtype=np.float64)[..., None, None] * f) * amplitude
    y = x.copy()
    re, im = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    z = (x[..., re] + 1j * x[..., im]) * turn
    y[..., re], y[..., im] = z.real, z.imag
    return y


def attend(q, keys, values, see, scale):
    """q [rows, D], keys / values [n, D], see [rows, n] truth values: (out [rows, D], lse [rows]); a row that sees nothing: 0, -inf."""
    q, keys, values = (np.asarray(a, dtype=np.float64) for a in (q, keys, values))
    out, lse = np.zeros((q.shape[0], values.shape[1])), np.full(q.shape[0], -np.inf)
    for r in range(q.shape[0]):
        idx = np.flatnonzero(see[r])
        if idx.size == 0:
            continue
        s = keys[idx] @ q[r] * scale
        m = s.max()
        w = np.exp(s - m)
        with np.errstate(invalid="ignore"):
            out[r] = (w @ values[idx]) / w.sum()
        lse[r] = m + np.log(w.sum())
    return out, lse


def visible(parents):
    """[T, T] truth values and depths [T] of a tree given by its nodes' parents (-1: node 0)."""
    T = len(parents)
    see, depth = np.zeros((T, T), dtype=bool), np.zeros(T, dtype=np.int32)
    for i, p in enumerate(parents):
        see[i, i] = True
        j = p
        while j >= 0:
            see[i, j] = True
            depth[i] += 1
            j = parents[j]
    return see, depth


class Cache:
    """Pages, owners and lengths, one call at a time; k and v [layers, pages, kv_heads, page_size, D]."""

    def __init__(self, k, v, table, seq_len, held, refs, max_nodes):
        self.k, self.v = np.array(k), np.array(v)
        self.table, self.len, self.held, self.refs = (np.array(a, dtype=np.int64) for a in (table, seq_len, held, refs))
        self.page, self.max_nodes, self.status = self.k.shape[3], max_nodes, OK

    def report(self, code):
        self.status = self.status or code

    def batch(self, slots, B=None):
        """(entry, slot) of the entries that count: padding left out, bad and repeated slots reported."""
        names = list(range(B)) if slots is None else [int(s) for s in slots]
        seen, got = set(), []
        for i, s in enumerate(names):
            if s == -1:
                continue
            if not 0 <= s < len(self.len) or s in seen:
                self.report(BAD_INDEX)
                continue
            seen.add(s)
            got.append((i, s))
        return got

    def pages_for(self, tokens):
        return -(-int(tokens) // self.page)

    def release(self, s, keep):
        for i in range(keep, self.held[s]):
            self.refs[self.table[s, i]] -= 1
            self.table[s, i] = -1
        self.held[s] = min(self.held[s], keep)

    def reserve(self, n, slots=None, B=None):
        entries = self.batch(slots, B)
        refs, plan = self.refs.copy(), []
        last_page = {}
        for _, s in entries:
            if self.len[s] + n > self.table.shape[1] * self.page:
                return self.report(PAGES)
            copy = False
            if self.len[s] % self.page:
                p = self.table[s, self.len[s] // self.page]
                copy = refs[p] - last_page.get(p, 0) > 1
                last_page[p] = last_page.get(p, 0) + 1
            plan.append((s, copy, max(self.pages_for(self.len[s] + n), self.held[s])))
        free = list(np.flatnonzero(self.refs == 0))
        if sum(int(c) + w - self.held[s] for s, c, w in plan) > len(free):
            return self.report(PAGES)
        for s, copy, want in plan:
            if copy:
                at, rows = self.len[s] // self.page, self.len[s] % self.page
                old, new = self.table[s, at], free.pop(0)
                for x in (self.k, self.v):
                    x[:, new, :, :rows] = x[:, old, :, :rows]
                self.refs[old] -= 1
                self.refs[new] = 1
                self.table[s, at] = new
            for i in range(self.held[s], want):
                self.table[s, i] = free.pop(0)
                self.refs[self.table[s, i]] = 1
            self.held[s] = want

    def row(self, s, token):
        return self.table[s, token // self.page], token % self.page

    def append(self, layer, k, v, slots=None, num_nodes=None):
        """k, v [B, T, kv_heads, D] as they are to be stored."""
        for i, s in self.batch(slots, k.shape[0]):
            for t in range(k.shape[1] if num_nodes is None else min(max(int(num_nodes[i]), 0), k.shape[1])):
                at = int(self.len[s]) + t
                if at // self.page >= self.held[s] or self.refs[self.table[s, at // self.page]] > 1:
                    self.report(BAD_INDEX)
                    continue
                p, r = self.row(s, at)
                self.k[layer, p, :, r], self.v[layer, p, :, r] = k[i, t], v[i, t]

    def owned(self, s, token):
        at = token // self.page
        return at < self.held[s] and self.refs[self.table[s, at]] <= 1

    def commit(self, accept, paths=None, slots=None, path_len=None):
        accept = np.asarray(accept).reshape(len(accept), -1)
        chosen = {}
        for i, s in self.batch(slots, accept.shape[0]):
            pick = int(accept[i].argmax())
            chosen[i] = pick
            length = paths.shape[2] if paths is not None else path_len
            a = min(max(int(accept[i, pick]), 0), length)
            base, before, kept = int(self.len[s]), 0, 0
            if not self.owned(s, base):
                a, kept = 0, -1
            for j in range(a):
                node = int(paths[i, pick, j]) if paths is not None else j + 1
                if node <= before or node >= self.max_nodes or not self.owned(s, base + node) or not self.owned(s, base + 1 + j):
                    break
                (fp, fr), (tp, tr) = self.row(s, base + node), self.row(s, base + 1 + j)
                for x in (self.k, self.v):
                    x[:, tp, :, tr] = x[:, fp, :, fr]
                before, kept = node, kept + 1
            if kept < a:
                self.report(BAD_INDEX)
            self.len[s] = base + kept + 1
            self.release(s, self.pages_for(self.len[s]))
        return chosen

    def fork(self, src, dst):
        used, srcs = set(), {int(s) for s, d in zip(src, dst) if int(d) != -1}
        for s, d in zip(map(int, src), map(int, dst)):
            if s == -1 or d == -1:
                continue
            n = len(self.len)
            if not (0 <= s < n and 0 <= d < n) or d in srcs or d in used or self.held[d] or self.len[d]:
                self.report(BAD_INDEX)
                used.add(d)
                continue
            used.add(d)
            keep = self.pages_for(self.len[s])
            self.table[d, :keep] = self.table[s, :keep]
            for p in self.table[s, :keep]:
                self.refs[p] += 1
            self.len[d], self.held[d] = self.len[s], keep

    def truncate(self, length=None, slots=None, B=None):
        for i, s in self.batch(slots, B if length is None else len(length)):
            to = 0 if length is None else int(length[i])
            if not 0 <= to <= self.len[s]:
                self.report(BAD_INDEX)
                continue
            self.len[s] = to
            self.release(s, self.pages_for(to))

    def compact(self):
        used = int((self.refs > 0).sum())
        holes, movers = np.flatnonzero(self.refs[:used] == 0), used + np.flatnonzero(self.refs[used:] > 0)
        renamed = np.arange(len(self.refs))
        for h, m in zip(holes, movers):
            for x in (self.k, self.v):
                x[:, h] = x[:, m]
            self.refs[h], self.refs[m] = self.refs[m], 0
            renamed[m] = h
        self.table = np.where(self.table >= 0, renamed[np.maximum(self.table, 0)], -1)
        return used

    def sequence(self, layer, head, s, extra=0):
        """Keys and values of a sequence's tokens and the `extra` rows behind them, cut to the pages held."""
        n = min(int(self.len[s]) + extra, int(self.held[s]) * self.page)
        pages = self.table[s, :self.pages_for(n)]
        D = self.k.shape[4]
        return tuple(x[layer, pages, head].reshape(-1, D)[:n] for x in (self.k, self.v))

    def attend(self, layer, q, see, scale, slots=None, num_nodes=None):
        """q [B, T, q_heads, D], see [T, T] or [B, T, T]: out and lse, NaN in rows that are not written."""
        B, T, Hq, D = q.shape
        H = self.k.shape[2]
        G = Hq // H
        out, lse = np.full(q.shape, np.nan), np.full(q.shape[:3], np.nan)
        for b in range(B):
            s = b if slots is None else int(slots[b])
            if not 0 <= s < len(self.len):
                if s != -1:
                    self.report(BAD_INDEX)
                continue
            nodes = T if num_nodes is None else min(max(int(num_nodes[b]), 0), T)
            m = see if see.ndim == 2 else see[b]
            for h in range(H):
                keys, values = self.sequence(layer, h, s, nodes)
                ctx = int(self.len[s])
                view = np.ones((nodes, len(keys)), dtype=bool)
                view[:, ctx:] = m[:nodes, :nodes][:, :max(0, len(keys) - ctx)]
                for g in range(G):
                    o, l = attend(q[b, :nodes, h * G + g], keys, values, view, scale)
                    out[b, :nodes, h * G + g], lse[b, :nodes, h * G + g] = o, l
        return out, lse
