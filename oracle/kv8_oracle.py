"""CPU oracle of the attention over prompts, the paged 8-bit cache and its page tables: plain numpy in fp64, one
sequence, head, block or request after the other, from the definitions in include/hgf.h."""
from __future__ import annotations

import math
from typing import List, Optional, Sequence, Tuple

import numpy as np

BLOCK = 16


# ------------------------------------------------------------------------------------- attention

def _weights(x: np.ndarray, seen: np.ndarray) -> np.ndarray:
    """softmax of a row over the keys that are seen; zeros where none is."""
    w = np.zeros_like(x)
    if seen.any():
        e = np.exp(x[seen] - x[seen].max())
        w[seen] = e / e.sum()
    return w


def attend(q, k, v, lam, seen, distance, softcap=0.0, slopes=None):
    """Rows of differential attention: q [n, 2H, d], k [m, 2H, d], v [m, H, d], seen and distance [n, m] -> [n, H, d].
    Keys that a row does not see do not enter its sums at all."""
    n, H2, d = q.shape
    H = H2 // 2
    q, k, v = (np.asarray(t, dtype=np.float64) for t in (q, k, v))
    out = np.zeros((n, H, d))
    for h in range(H):
        for i in range(n):
            at = np.nonzero(seen[i])[0]
            if len(at) == 0:
                continue
            a = []
            for g in (h, H + h):
                x = k[at, g] @ q[i, g] / math.sqrt(d)
                if softcap > 0:
                    x = softcap * np.tanh(x / softcap)
                if slopes is not None:
                    x = x - float(slopes[g]) * distance[i, at]
                a.append(_weights(x, np.ones(len(at), dtype=bool)) @ v[at, h])
            out[i, h] = 0.5 * (a[0] - lam * a[1])
    return out


def prefill(q, k, v, cu_q, lam, cu_k=None, causal=True, prefix=None, doc_q=None, doc_k=None, softcap=0.0, slopes=None):
    """[Tq, H, d] in fp64; rows of no sequence are NaN (a caller's are left as they were)."""
    cu_k = cu_q if cu_k is None else cu_k
    out = np.full((q.shape[0], v.shape[1], q.shape[2]), np.nan)
    for b in range(len(cu_q) - 1):
        nq, nk = cu_q[b + 1] - cu_q[b], cu_k[b + 1] - cu_k[b]
        if nq <= 0:
            continue
        qs, ks = slice(cu_q[b], cu_q[b + 1]), slice(cu_k[b], cu_k[b] + max(nk, 0))
        p, j = nk - nq + np.arange(nq)[:, None], np.arange(max(nk, 0))[None, :]
        seen = np.ones((nq, max(nk, 0)), dtype=bool)
        if causal:
            seen = j <= p
            if prefix is not None:
                seen = seen | (j < prefix[b])
        if doc_q is not None:
            dq, dk = np.asarray(doc_q)[qs][:, None], np.asarray(doc_k)[ks][None, :]
            seen = seen & (dq == dk) & (dk >= 0)
        out[qs] = attend(q[qs], k[ks], v[ks], lam, seen, np.abs(p - j), softcap, slopes)
    return out


# ------------------------------------------------------------------------------------- the cache

def block_exponent(amax: float) -> int:
    """The smallest e >= -30 with 127 * 2^e >= amax."""
    e = -30
    while 127.0 * 2.0 ** e < amax:
        e += 1
    return e


def storable(x: np.ndarray) -> np.ndarray:
    x = np.asarray(x, dtype=np.float64)
    return np.clip(np.where(np.isnan(x), 0.0, x), -65504.0, 65504.0)


class Pool:
    """Codes [n_pages, heads, page, d] and scales [n_pages, heads, page / 16] of K or V."""

    def __init__(self, n_pages: int, page: int, heads: int, d: int):
        self.page = page
        self.codes = np.zeros((n_pages, heads, page, d), dtype=np.int64)
        self.scale = np.zeros((n_pages, heads, page // BLOCK), dtype=np.float64)

    def write(self, row: Sequence[int], start: int, x: np.ndarray) -> None:
        """Tokens x [n, heads, d] at positions start .. of the sequence whose pages are `row` (missing pages: dropped)."""
        x = storable(x)
        end = start + len(x)
        for first in range(max(start, 0) // BLOCK * BLOCK, end, BLOCK):
            pg = row[first // self.page] if first // self.page < len(row) else -1
            if not 0 <= pg < len(self.codes):
                continue
            lo, hi = max(start, 0, first), min(end, first + BLOCK)
            off, blk = first % self.page, first % self.page // BLOCK
            for h in range(x.shape[1]):
                new = x[lo - start:hi - start, h]
                s = 2.0 ** block_exponent(np.abs(new).max())
                before = lo - first
                if before:
                    old = self.scale[pg, h, blk]
                    s = max(s, old)
                    part = self.codes[pg, h, off:off + before]
                    part[:] = np.clip(np.rint(part * (old / s)), -127, 127)
                self.codes[pg, h, off + before:off + hi - first] = np.clip(np.rint(new / s), -127, 127)
                self.scale[pg, h, blk] = s

    def read(self, row: Sequence[int], positions) -> np.ndarray:
        """[n, heads, d] fp64; zeros where there is no such position or page."""
        out = np.zeros((len(positions), self.codes.shape[1], self.codes.shape[3]))
        for i, p in enumerate(positions):
            pg = row[p // self.page] if p >= 0 and p // self.page < len(row) else -1
            if 0 <= pg < len(self.codes):
                out[i] = self.codes[pg, :, p % self.page] * self.scale[pg, :, p % self.page // BLOCK, None]
        return out

    def copy(self, pairs) -> None:
        n = len(self.codes)
        for a, b in pairs:
            if 0 <= a < n and 0 <= b < n and a != b:
                self.codes[b], self.scale[b] = self.codes[a], self.scale[a]


def decode(q, k: Pool, v: Pool, table, lens, rows, lam, softcap=0.0, slopes=None):
    """[B, H, d] fp64: row b is sequence rows[b], its newest token attends to all positions that have a page."""
    out = np.zeros((len(rows), v.codes.shape[1], q.shape[2]))
    for i, s in enumerate(rows):
        if not 0 <= s < len(table):
            continue
        n = min(max(int(lens[s]), 0), table.shape[1] * k.page)
        if n == 0:
            continue
        there = np.array([0 <= table[s][p // k.page] < len(k.codes) for p in range(n)])
        kk, vv = k.read(table[s], range(n)), v.read(table[s], range(n))
        out[i] = attend(q[i:i + 1], kk, vv, lam, there[None, :], (n - 1 - np.arange(n))[None, :], softcap, slopes)[0]
    return out


# ------------------------------------------------------------------------------------- pages

class Pages:
    """Table, lengths and counts; every request of a list after the other."""

    def __init__(self, n_pages: int, page: int, n_seqs: int, max_pages: int):
        self.page = page
        self.table = np.full((n_seqs, max_pages), -1, dtype=np.int64)
        self.lens, self.refs = np.zeros(n_seqs, dtype=np.int64), np.zeros(n_pages, dtype=np.int64)

    def _need(self, n: int) -> int:
        return (n + self.page - 1) // self.page

    def _serve(self, wants: List[Optional[int]]) -> Tuple[List[bool], List[List[int]]]:
        """Which requests are granted, and their pages: the lowest free ones in order; once the pages do not reach, only
        requests that need none are granted."""
        free = [int(p) for p in np.nonzero(self.refs == 0)[0]]
        asked, ok, pages = 0, [], []
        for w in wants:
            asked += w or 0
            yes = w is not None and (w == 0 or asked <= len(free))
            ok.append(yes)
            pages.append(free[asked - w:asked] if yes else [])
        return ok, pages

    def grow(self, seqs, new):
        seen, wants = set(), []
        for s, a in zip(seqs, new):
            bad = not 0 <= s < len(self.lens) or s in seen
            if 0 <= s < len(self.lens):
                bad = bad or a < 0 or self.lens[s] + a > self.table.shape[1] * self.page
                seen.add(s)
            wants.append(None if bad else self._need(self.lens[s] + a) - self._need(self.lens[s]))
        ok, pages = self._serve(wants)
        for s, a, yes, got in zip(seqs, new, ok, pages):
            if yes:
                at = self._need(self.lens[s])
                self.table[s, at:at + len(got)] = got
                self.refs[got] = 1
                self.lens[s] += a
        return np.array(ok, dtype=np.int64)

    def fork(self, src, dst):
        seen, wants = set(), []
        for s, d in zip(src, dst):
            bad = not 0 <= s < len(self.lens) or not 0 <= d < len(self.lens) or s == d or d in seen
            bad = bad or self.lens[d] != 0
            seen.add(d)
            wants.append(None if bad else int(self.lens[s] % self.page != 0))
        ok, pages = self._serve(wants)
        pairs = np.full((len(src), 2), -1, dtype=np.int64)
        table, lens = self.table.copy(), self.lens.copy()             # (sources are what they were before the call)
        for i, (s, d, yes, got) in enumerate(zip(src, dst, ok, pages)):
            if yes:
                full = lens[s] // self.page
                self.table[d, :full] = table[s, :full]
                self.refs[table[s, :full]] += 1
                if got:
                    pairs[i] = table[s, full], got[0]
                    self.table[d, full], self.refs[got[0]] = got[0], 1
                self.lens[d] = lens[s]
        return pairs, np.array(ok, dtype=np.int64)

    def free(self, seqs):
        for s in set(int(x) for x in seqs if 0 <= x < len(self.lens)):
            used = self._need(self.lens[s])
            for pg in self.table[s, :used]:
                self.refs[pg] -= 1
            self.table[s, :used] = -1
            self.lens[s] = 0

    def compact(self):
        live = int((self.refs > 0).sum())
        holes = [p for p in range(live) if self.refs[p] == 0]
        movers = [p for p in range(live, len(self.refs)) if self.refs[p] > 0]
        pairs = np.full((max(1, len(self.refs) // 2), 2), -1, dtype=np.int64)
        moved = np.where(self.refs > 0, np.arange(len(self.refs)), -1)
        for i, (a, b) in enumerate(zip(movers, holes)):
            pairs[i] = a, b
            moved[a] = b
            self.refs[b], self.refs[a] = self.refs[a], 0
        for s in range(len(self.lens)):
            used = self._need(self.lens[s])
            self.table[s, :used] = moved[self.table[s, :used]]
        return pairs, len(movers), moved
