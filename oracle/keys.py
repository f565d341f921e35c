"""fp64 NumPy oracle of attention over keys that are not the queries' own: the cache with a scale per page and head, attention over
cached or given keys, and the pool of pages.

Written from the definitions, with loops where a loop is plainest; shares no code with the library or with the measured cases.
"""
import numpy as np

from .layer import e4m3_bytes, e4m3_values, f32


def append(codes, scale, x, table, lengths, counts, page):
    """x [B,H,T,d] behind the sequences' tokens; codes [pages,H,page,d] bytes and scale [pages,H] float64 are changed in place."""
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        for b in range(x.shape[0]):
            end = lengths[b] + counts[b]
            for place in range(lengths[b] // page, -(-end // page)):
                i = table[b][place] if place < len(table[b]) else -1
                lo, hi = max(lengths[b] - place * page, 0), min(end - place * page, page)
                if lo >= hi or not 0 <= i < codes.shape[0]:
                    continue
                first = place * page - lengths[b]
                for h in range(x.shape[1]):
                    new = x[b, h, first + lo:first + hi]
                    held = scale[i, h] if lo else 0.0
                    fresh = float(f32(np.abs(new).max() / 448.0))
                    now = fresh + held if np.isnan(fresh + held) else max(fresh, held)
                    if now > held and lo:
                        codes[i, h, :lo] = e4m3_bytes(f32(e4m3_values(codes[i, h, :lo]) * f32(held / now)))
                    codes[i, h, lo:hi] = e4m3_bytes(f32(new / now)) if now != 0 else 0
                    scale[i, h] = now


def gathered(codes, scale, table, length, page):
    """[H, length, d] values of a sequence; rows on pages that are named wrongly are NaN."""
    out = np.full((codes.shape[1], length, codes.shape[3]), np.nan)
    for n in range(length):
        i = table[n // page] if n // page < len(table) else -1
        if 0 <= i < codes.shape[0]:
            out[:, n] = e4m3_values(codes[i, :, n % page]) * scale[i][:, None]
    return out


def attention(q, k, v, there, scale):
    """q [T,d], k, v [S,d], there [T,S] or [S]: (o, lse, the weights' mean magnitude of v per output, the largest sum |q||k| scale)."""
    there = np.broadcast_to(there, (q.shape[0], k.shape[0]))
    o, lse, size = np.zeros_like(q), np.full(q.shape[0], -np.inf), np.zeros_like(q)
    for t in range(q.shape[0]):
        on = np.flatnonzero(there[t])
        if on.size == 0:
            continue
        x = k[on] @ q[t] * scale
        top = x.max()
        p = np.exp(x - top)
        lse[t] = top + np.log(p.sum())
        o[t], size[t] = p @ v[on] / p.sum(), p @ np.abs(v[on]) / p.sum()
    used = np.flatnonzero(there.any(0))
    sums = np.abs(q) @ np.abs(k[used]).T * scale if used.size else np.zeros((1, 1))
    return o, lse, size, sums.max(initial=0.0)


class Pool:
    """The pool of pages, entry by entry: refs, table and lengths are lists that the calls change; `moved` lists (source, destination)."""

    def __init__(self, refs, table, lengths, page):
        self.refs, self.table, self.lengths, self.page, self.moved, self.short = list(refs), [list(r) for r in table], list(lengths), page, [], False

    def lowest(self):
        for i, r in enumerate(self.refs):
            if r <= 0:
                self.refs[i] = 1
                return i
        self.short = True
        return -1

    def take(self, counts):
        for b, row in enumerate(self.table):
            for e in range(-(-self.lengths[b] // self.page), -(-(self.lengths[b] + counts[b]) // self.page)):
                row[e] = self.lowest()

    def fork(self, parents, children):
        own = []
        for p, c in zip(parents, children):
            part = self.lengths[p] % self.page != 0
            own.append(self.lowest() if part else None)
        for p, c, i in zip(parents, children, own):
            full = self.lengths[p] // self.page
            self.lengths[c] = self.lengths[p]
            self.table[c] = self.table[p][:full] + [-1] * (len(self.table[p]) - full)
            for j in self.table[p][:full]:
                self.refs[j] += 1
            if i is not None:
                self.table[c][full] = i
                if i < 0:
                    self.lengths[c] = full * self.page
                else:
                    self.moved.append((self.table[p][full], i))

    def free(self, rows, keep):
        for r, n in zip(rows, keep):
            for e in range(-(-n // self.page), len(self.table[r])):
                if self.table[r][e] >= 0:
                    self.refs[self.table[r][e]] -= 1
                    self.table[r][e] = -1
            self.lengths[r] = min(self.lengths[r], n)

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        holes = [i for i in range(live) if self.refs[i] <= 0]
        movers = [i for i in range(live, len(self.refs)) if self.refs[i] > 0]
        to = dict(zip(movers, holes))
        for a, b in to.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
            self.moved.append((a, b))
        self.table = [[to.get(i, i) for i in row] for row in self.table]
        return live
