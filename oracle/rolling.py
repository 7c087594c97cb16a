"""Plain statements of the operators of a rolling paged cache, one step after the other: attention with a window and sinks,
rotary positions, and the calls on pages.  As in the rest of the oracle nothing here is shared with the CUDA package."""
from __future__ import annotations

import numpy as np


# ---------------------------------------------------------------------------------- attention
def window_keys(position: int, window: int, n_sinks: int) -> list[int]:
    """The keys that the query at `position` sees."""
    return [j for j in range(position + 1) if position - j < window or j < n_sinks]


def attention_window(q: np.ndarray, k: np.ndarray, v: np.ndarray, kv_len: int, window: int, n_sinks: int, sm_scale: float):
    """q [n_q][Hq][D], k and v [Hkv][>= kv_len][D], float64.  Returns (out [n_q][Hq][D], lse [n_q][Hq])."""
    n_q, hq, d = q.shape
    group = hq // k.shape[0]
    out = np.zeros((n_q, hq, d))
    lse = np.full((n_q, hq), -np.inf)
    for t in range(n_q):
        keys = window_keys(kv_len - n_q + t, window, n_sinks)
        if not keys:
            continue
        for h in range(hq):
            x = sm_scale * (k[h // group][keys] @ q[t, h])
            m = x.max()
            e = np.exp(x - m)
            out[t, h] = (e @ v[h // group][keys]) / e.sum()
            lse[t, h] = m + np.log(e.sum())
    return out, lse


# ---------------------------------------------------------------------------------- rotary positions
def frequencies(rot_dim: int, base: float) -> np.ndarray:
    return np.array([base ** (-2.0 * i / rot_dim) for i in range(rot_dim // 2)])


def rotate(x: np.ndarray, positions, freq: np.ndarray, factor: float, interleaved: bool, sections=None) -> np.ndarray:
    """x [..., D] float64; positions: one a position axis.  The angle is taken modulo a turn in extended precision."""
    rot = 2 * len(freq)
    y = np.array(x, dtype=np.float64)
    axis = [a for a, n in enumerate(sections or (len(freq),)) for _ in range(n)]
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        angle = float(np.fmod(np.longdouble(positions[axis[i]]) * np.longdouble(freq[i]), 2 * np.arctan2(np.longdouble(0), np.longdouble(-1))))
        c, s = factor * np.cos(angle), factor * np.sin(angle)
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


# ---------------------------------------------------------------------------------- pages
class Pool:
    """The counts of a pool of pages and the calls on block tables (lists of lists, -1: unmapped)."""

    def __init__(self, n_pages: int, page: int):
        self.ref, self.page = [0] * n_pages, page

    def reserve(self, table, lens, new, max_len):
        """Returns (copies [(source, destination, rows)], ok, refused sequences)."""
        before, refused, wanted = list(self.ref), [], []
        held = list(self.ref)                                  # less the sequences that have already left a begun page
        for b, (n, m) in enumerate(zip(lens, new)):
            if n < 0 or m < 0 or n > max_len or n + m > max_len:
                refused.append(b)
                continue
            if m == 0:
                continue
            for j in range(n // self.page, (n + m - 1) // self.page + 1):
                at = table[b][j]
                if not 0 <= at < len(self.ref):
                    wanted.append((b, j, -1, 0))
                elif j == n // self.page and n % self.page:
                    if held[at] > 1:
                        wanted.append((b, j, at, n % self.page))
                        held[at] -= 1
                    else:
                        held[at] -= 1                          # its own now
                elif before[at] > 1:
                    wanted.append((b, j, at, 0))
        free = [n for n, r in enumerate(before) if r == 0]
        if len(wanted) > len(free):
            return [], False, refused
        copies = []
        for (b, j, old, rows), n in zip(wanted, free):
            table[b][j] = n
            self.ref[n] = 1
            if old >= 0:
                self.ref[old] -= 1
            if rows:
                copies.append((old, n, rows))
        return copies, True, refused

    def release(self, table, lens, window, n_sinks):
        for b, n in enumerate(lens):
            for j, at in enumerate(table[b]):
                if any(r < n and (r < n_sinks or r >= n - window) for r in range(j * self.page, (j + 1) * self.page)):
                    continue
                if 0 <= at < len(self.ref):
                    self.ref[at] -= 1
                table[b][j] = -1

    def fork(self, table, lens, parents):
        new_table, new_lens = [], []
        for p in parents:
            kept = -(-lens[p] // self.page) if p >= 0 else 0
            row = [at if j < kept and 0 <= at < len(self.ref) else -1 for j, at in enumerate(table[p])] if p >= 0 else [-1] * len(table[0])
            for at in row:
                if at >= 0:
                    self.ref[at] += 1
            new_table.append(row)
            new_lens.append(lens[p] if p >= 0 else 0)
        for row in table:
            for at in row:
                if 0 <= at < len(self.ref):
                    self.ref[at] -= 1
        return new_table, new_lens

    def compact(self, table):
        """Returns (moves [(source, destination)], pages in use)."""
        n_used = sum(r > 0 for r in self.ref)
        holes = [n for n in range(n_used) if self.ref[n] == 0]
        movers = [n for n in range(n_used, len(self.ref)) if self.ref[n] > 0]
        to = dict(zip(movers, holes))
        for src, dst in to.items():
            self.ref[dst], self.ref[src] = self.ref[src], 0
        for row in table:
            for j, at in enumerate(row):
                row[j] = to.get(at, at)
        return list(to.items()), n_used
