"""Plain oracle of the rotary positions and of the paged window memory.

Python integers and NumPy in fp64, written from the definitions, token by
token; no code shared with the library.

* rotary_apply: pair p of a head turns by pos[axis(p)] * freq[p];
* PagedOracle: which tokens a sequence holds, which pages they lie in, and
  which keys a query sees: token p in block b = p // B sees held tokens of
  blocks <= b that are among the first `sinks` blocks or the last `window`
  blocks up to b (window 0: all).
"""
from __future__ import annotations

from typing import List, Sequence

import numpy as np


def rotary_apply(x: np.ndarray, pos: np.ndarray, pairs: Sequence[int], theta: float, layout: str = "interleaved",
                 inverse: bool = False) -> np.ndarray:
    """x [rows][heads][D] (fp64), pos [rows][3]; unrounded."""
    y = np.array(x, dtype=np.float64, copy=True)
    half = x.shape[-1] // 2
    p = 0
    for axis in range(3):
        for k in range(pairs[axis]):
            ang = pos[:, axis].astype(np.float64) * float(theta) ** (-k / pairs[axis])
            c, s = np.cos(ang)[:, None], np.sin(ang)[:, None] * (-1.0 if inverse else 1.0)
            i, j = (2 * p, 2 * p + 1) if layout == "interleaved" else (p, p + half)
            a, b = x[..., i].astype(np.float64), x[..., j].astype(np.float64)
            y[..., i], y[..., j] = a * c - b * s, a * s + b * c
            p += 1
    return y


class PagedOracle:
    OK, EINVAL, ESTATE, ENOMEM = 0, -1, -2, -3

    def __init__(self, seqs: int, pages: int, page_tokens: int, max_tokens: int, block: int = 1, window: int = 0,
                 sinks: int = 0, grid=(1, 1)):
        self.seqs, self.n_pages, self.P, self.max_tokens = seqs, pages, page_tokens, max_tokens
        self.B, self.W, self.S, self.grid = block, window, sinks if window else 0, grid
        self.held = [0] * seqs
        self.table: List[dict] = [dict() for _ in range(seqs)]  # page index -> page
        self.given_up = [0] * seqs   # pages below this index, behind the sinks', were given back

    def window_low(self, p: int) -> int:
        return 0 if self.W == 0 else max(0, p // self.B - self.W + 1) * self.B

    def sees(self, p: int, held: int) -> np.ndarray:
        """Keys that the query at position p sees, in order."""
        j = np.arange(held)
        b, jb = p // self.B, j // self.B
        ok = jb <= b
        if self.W:
            ok &= (jb > b - self.W) | (jb < self.S)
        return j[ok]

    def _pages(self, kept: int, end: int) -> set:
        """Page indices a sequence keeps for tokens [0, end), its new ones starting at `kept`."""
        front = -(-(self.S * self.B) // self.P)
        low = self.window_low(kept) // self.P
        return {i for i in range(-(-end // self.P)) if i < front or i >= low}

    def plan(self, kept: Sequence[int], added: Sequence[int], rows: int, max_new: int) -> dict:
        front = -(-(self.S * self.B) // self.P)
        status, q_start, at = [self.OK] * self.seqs, [], 0
        for s in range(self.seqs):
            k, n = kept[s], added[s]
            q_start.append(min(at, rows))
            at += max(n, 0)
            if k < 0 or n < 0 or n > max_new or k > self.held[s] or k + n > self.max_tokens or (n > 0 and at > rows):
                status[s] = self.EINVAL
            elif self.given_up[s] > front and k > front * self.P and self.window_low(k) // self.P < self.given_up[s]:
                status[s] = self.ESTATE
        q_start.append(min(at, rows))
        ok = [s for s in range(self.seqs) if status[s] == self.OK]
        # Every admitted sequence gives back first; then pages go out in order until one does not fit.
        free = self.free_pages()
        n_free = len(free)
        keep, need = {}, {}
        for s in ok:
            want = self._pages(kept[s], kept[s] + added[s])
            mapped = self._mapped_after_going_back(s, kept[s], front)
            keep[s], need[s] = want & mapped, len(want - mapped)
            n_free += len(self.table[s]) - len(keep[s])
        full = False
        for s in ok:
            if need[s] > 0 and (full or need[s] > n_free):
                status[s], full = self.ENOMEM, True
            else:
                n_free -= need[s]
        for s in ok:
            end = kept[s] + (added[s] if status[s] == self.OK else 0)
            want = self._pages(kept[s], end) & self._mapped_after_going_back(s, kept[s], front)
            self.table[s] = {i: p for i, p in self.table[s].items() if i in want}
            self.given_up[s] = max(front, self.window_low(kept[s]) // self.P)
            self.held[s] = end
        pool = iter(sorted(self.free_pages()))
        for s in ok:
            if status[s] == self.OK:
                for i in sorted(self._pages(kept[s], self.held[s]) - set(self.table[s])):
                    self.table[s][i] = next(pool)
        slots, pos = [-1] * rows, [(0, 0, 0)] * rows
        gh, gw = self.grid
        for s in range(self.seqs):
            if status[s] == self.OK:
                for i in range(added[s]):
                    p = kept[s] + i
                    slots[q_start[s] + i] = self.table[s][p // self.P] * self.P + p % self.P
                    pos[q_start[s] + i] = (p // (gh * gw), p % (gh * gw) // gw, p % gw)
        return dict(q_start=q_start, status=status, slots=slots, pos=pos, held=list(self.held),
                    free=len(self.free_pages()))

    def _mapped_after_going_back(self, s: int, kept: int, front: int) -> set:
        """Pages of s that are still good when it goes back to `kept` tokens: none behind the sinks if all that is
        kept lies in the sinks' pages and some pages behind them were given back."""
        mapped = set(self.table[s])
        if self.given_up[s] > front and kept <= front * self.P:
            mapped = {i for i in mapped if i < front}
        return mapped

    def free_pages(self) -> list:
        used = {p for t in self.table for p in t.values()}
        return [p for p in range(self.n_pages) if p not in used]

    def table_rows(self) -> np.ndarray:
        width = -(-self.max_tokens // self.P)
        out = np.full((self.seqs, width), -1, dtype=np.int64)
        for s, t in enumerate(self.table):
            for i, p in t.items():
                out[s, i] = p
        return out


def paged_attend(q: np.ndarray, keys: np.ndarray, values: np.ndarray, positions: Sequence[int], oracle: PagedOracle,
                 scale=None):
    """Attention of one sequence's queries q [n][H][D] at `positions` over its tokens' keys and values [held][Hk][D].
    Returns O, LSE [H][n] and the weighted mean of |V| (what a relative error of the weights is relative to)."""
    n, H, D = q.shape
    G = H // keys.shape[1]
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    O, A, L = np.zeros((n, H, D)), np.zeros((n, H, D)), np.full((H, n), -np.inf)
    for i, p in enumerate(positions):
        j = oracle.sees(p, len(keys))
        if len(j) == 0:
            continue
        for h in range(H):
            s = scale * (keys[j, h // G] @ q[i, h])
            m = s.max()
            w = np.exp(s - m)
            v = values[j, h // G]
            O[i, h], A[i, h] = w @ v / w.sum(), w @ np.abs(v) / w.sum()
            L[h, i] = m + np.log(w.sum())
    return O, L, A
