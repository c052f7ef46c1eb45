"""Plain host forms of the paged-pool calls and of the attention over paged sequences (numpy, 64 bits).

The pool calls are written as the header states them: entries in list order, lowest free page first, one entry at a time.
"""
from __future__ import annotations

import math

import numpy as np

OK, INVALID, BAD_STATE, OOM = 0, -1, -2, -3


class HostPool:
    """Mirror of a pool: ``k``, ``v`` [layers][pages][page][heads * head_dim] as 16-bit patterns, tables as int32."""

    def __init__(self, k, v, table, length, refs):
        self.k, self.v = (x.reshape(x.shape[0], x.shape[1], x.shape[2], -1).copy() for x in (k, v))
        self.table, self.len, self.refs = table.copy(), length.copy(), refs.copy()
        self.page, self.max_pages = k.shape[2], table.shape[1]

    def pages(self, rows):
        return -(-int(rows) // self.page)

    def _slot(self, s):
        return 0 <= s < len(self.len)

    def _sound(self, s):
        if not 0 <= self.len[s] <= self.max_pages * self.page:
            return False
        t = self.table[s, :self.pages(self.len[s])]
        return bool(np.all((t >= 0) & (t < len(self.refs))))

    def _release(self, s, first=0):
        for j in range(first, self.pages(self.len[s])):
            self.refs[self.table[s, j]] -= 1
            self.table[s, j] = -1

    def _take(self, needs):
        """Pages for each need in order; None where they do not suffice (then nothing later is granted either)."""
        free = [int(p) for p in np.nonzero(self.refs == 0)[0]]
        out, at = [], 0
        for n in needs:
            out.append(free[at:at + n] if at + n <= len(free) else (None if n else []))
            at += n
        for got in out:
            for p in got or []:
                self.refs[p] = 1
        return out

    def resize(self, seqs, lens):
        refs0 = self.refs.copy()
        st, todo, seen = [], [], set()
        for s, n in zip(seqs, lens):
            code = OK
            if not self._slot(s) or s in seen:
                code = INVALID
            elif not self._sound(s):
                code = BAD_STATE
            elif not 0 <= n <= self.max_pages * self.page:
                code = INVALID
            elif n < self.len[s] and n % self.page and refs0[self.table[s, n // self.page]] > 1:
                code = BAD_STATE
            seen.add(s)
            st.append(code)
        for s, n, c in zip(seqs, lens, st):
            if c == OK and self.pages(n) < self.pages(self.len[s]):
                self._release(s, self.pages(n))
        got = self._take([max(0, self.pages(n) - self.pages(self.len[s])) if c == OK else 0 for s, n, c in zip(seqs, lens, st)])
        for i, (s, n) in enumerate(zip(seqs, lens)):
            if st[i] != OK:
                continue
            if got[i] is None:
                st[i] = OOM
                continue
            had = self.pages(self.len[s])
            self.table[s, had:had + len(got[i])] = got[i]
            self.len[s] = n
        return st

    def _place(self, src, dst, st, keeps, deep):
        """fork and compact: dst holds rows keeps[i] of src; ``deep``: nothing is shared."""
        old = {i: self.table[s].copy() for i, s in enumerate(src) if st[i] == OK}
        shared = {}
        for i in old:
            lead = next((t for t, x in enumerate(keeps[i]) if x != t), len(keeps[i]))
            shared[i] = 0 if deep else lead // self.page
        for i in old:
            if dst[i] != src[i]:
                self._release(dst[i])
        got = self._take([self.pages(len(keeps[i])) - shared[i] if i in old else 0 for i in range(len(src))])
        moves = []
        for i in old:
            s, d = src[i], dst[i]
            if got[i] is None:
                st[i] = OOM
                if d != s:
                    self.len[d] = 0
                continue
            new = list(old[i][:shared[i]]) + got[i]
            if d == s:
                for p in old[i][shared[i]:self.pages(self.len[s])]:
                    self.refs[p] -= 1
            else:
                for p in new[:shared[i]]:
                    self.refs[p] += 1
            moves.append((i, new))
        k0, v0 = self.k.copy(), self.v.copy()
        for i, new in moves:
            d, P = dst[i], self.page
            self.table[d] = -1
            self.table[d, :len(new)] = new
            self.len[d] = len(keeps[i])
            for x in range(shared[i] * P, len(keeps[i])):
                y = keeps[i][x]
                self.k[:, new[x // P], x % P] = k0[:, old[i][y // P], y % P]
                self.v[:, new[x // P], x % P] = v0[:, old[i][y // P], y % P]
        return st

    def fork(self, src, dst, deep):
        st, seen = [], set()
        for s, d in zip(src, dst):
            code = OK
            if not self._slot(s) or not self._slot(d) or d in seen or d in src:
                code = INVALID
            elif not self._sound(s) or not self._sound(d):
                code = BAD_STATE
            seen.add(d)
            st.append(code)
        return self._place(src, dst, st, [range(self.len[s]) if c == OK else [] for s, c in zip(src, st)], deep)

    def compact(self, src, dst, keeps):
        st, seen = [], set()
        for i, (s, d) in enumerate(zip(src, dst)):
            code = OK
            if not self._slot(s) or not self._slot(d) or d in seen or any(x == d and y != x for x, y in zip(src, dst)):
                code = INVALID
            elif not self._sound(s) or not self._sound(d):
                code = BAD_STATE
            elif any(not 0 <= x < self.len[s] for x in keeps[i]) or any(b <= a for a, b in zip(keeps[i], keeps[i][1:])):
                code = INVALID
            seen.add(d)
            st.append(code)
        return self._place(src, dst, st, keeps, False)

    def write(self, layer, seqs, start, row_ptr, k_rows, v_rows):
        st, seen = [], set()
        for i, s in enumerate(seqs):
            n = row_ptr[i + 1] - row_ptr[i]
            code = OK
            if not self._slot(s) or s in seen or n < 0 or row_ptr[i] < 0 or row_ptr[i + 1] > len(k_rows):
                code = INVALID
            elif not 0 <= self.len[s] <= self.max_pages * self.page:
                code = BAD_STATE
            else:
                at = self.len[s] - n if start is None else start[i]
                if at < 0 or at + n > self.len[s]:
                    code = INVALID
                else:
                    t = self.table[s, at // self.page:self.pages(at + n)] if n else []
                    if any(not 0 <= p < len(self.refs) or self.refs[p] != 1 for p in t):
                        code = BAD_STATE
            if code == OK:
                for x in range(n):
                    p = self.table[s, (at + x) // self.page]
                    self.k[layer, p, (at + x) % self.page] = k_rows[row_ptr[i] + x]
                    self.v[layer, p, (at + x) % self.page] = v_rows[row_ptr[i] + x]
            seen.add(s)
            st.append(code)
        return st


def attention(k, v, q, n, nq, ratio, scale, half):
    """One sequence: k, v [n][kv_heads][d], q [nq][heads][d], 64 bits.  Returns out, lse and bounds on the error of each.

    Bounds.  half: half a step of the 16-bit type.  The weights are rounded to it for the product with V and the result is rounded
    once: half * sum p|v| + half * |o|.  A score is a sum of d products in fp32 (at most 2^-23 of the sum of magnitudes a term), scaled
    (2 roundings, magnified by the size of the score) and put through an exponential of relative error 2^-22 or less; the sum of n
    weights adds n 2^-24 at most, every joining of pieces a few roundings more.
    """
    heads, d = q.shape[1], q.shape[2]
    out, lse = np.zeros((nq, heads, d)), np.full((nq, heads), -np.inf)
    eo, el = np.zeros((nq, heads, d)), np.zeros((nq, heads))
    for j in range(nq):
        m = n - nq + j + 1
        if m <= 0:
            continue
        for h in range(heads):
            with np.errstate(invalid="ignore", over="ignore"):
                kh, vh = k[:m, h // ratio], v[:m, h // ratio]
                s = kh @ q[j, h] * scale
                big = np.max(np.abs(kh) @ np.abs(q[j, h])) * abs(scale)
                lse[j, h] = s.max() + math.log(np.sum(np.exp(s - s.max())))
                p = np.exp(s - lse[j, h])
                out[j, h] = p @ vh
                rel = 2 * (d + 4) * 2.0 ** -23 * big + 2.0 ** -21 + m * 2.0 ** -24 + 64 * 2.0 ** -24
                a = p @ np.abs(vh)
                eo[j, h] = (half + 2 * rel) * a + half * np.abs(out[j, h]) + 1e-30
                el[j, h] = rel + 2.0 ** -22 * (abs(lse[j, h]) + 1)
    return out, lse, eo, el
