"""The operators between two model calls in float64, from their definitions: rotary positions with several axes,
acceptance of drafted tokens, kept rows, the pages of a pool, low-rank adapters.  Nothing here is shared with the GPU path.
"""
from __future__ import annotations

import numpy as np

from . import cache as oc

F64 = np.float64
PAGE = 16


# ----------------------------------------------------------------------------- rotary positions with several axes
def pair_axes(pairs, cyclic=False):
    """The axis of every pair: runs in order, or dealt one by one to the axes that have not got theirs."""
    if not cyclic:
        return np.repeat(np.arange(len(pairs)), pairs)
    left, out = list(pairs), []
    while any(left):
        for a in range(len(left)):
            if left[a]:
                out.append(a)
                left[a] -= 1
    return np.array(out, int)


def axes_frequencies(pairs, theta, cyclic=False, own_freqs=False, **scaling):
    """Radians per position of every pair (``scaling`` as for ``oc.rope_frequencies``)."""
    half = sum(pairs)
    if not own_freqs:
        return oc.rope_frequencies(2 * half, theta, **scaling)
    axis, f = pair_axes(pairs, cyclic), np.zeros(half)
    for a, m in enumerate(pairs):
        if m:
            f[axis == a] = oc.rope_frequencies(2 * m, theta, **scaling)
    return f


def rotate_axes(x, pos, pairs, freq, cyclic=False, interleaved=False, mscale=1.0):
    """The first 2 sum(pairs) dimensions of rows [n, heads, D] turned by pos[axis of the pair] [axes, n]."""
    y = np.array(x, F64)
    rot = 2 * sum(pairs)
    if rot == 0:
        return y
    ang = np.asarray(pos, F64)[pair_axes(pairs, cyclic)].T * freq                    # [n, half]
    c, s = np.cos(ang)[:, None] * mscale, np.sin(ang)[:, None] * mscale
    a = slice(0, rot, 2) if interleaved else slice(0, rot // 2)
    b = slice(1, rot, 2) if interleaved else slice(rot // 2, rot)
    ya, yb = y[..., a].copy(), y[..., b].copy()
    y[..., a] = ya * c - yb * s
    y[..., b] = yb * c + ya * s
    return y


# ----------------------------------------------------------------------------- acceptance
def weights(logits, t):
    """Probabilities of a row at temperature t times a factor that makes the largest 1; None where there are none.  (Not
    normalised: equal logits have weights of exactly 1, whose running sums are exact, so that a number on a border
    between two of them decides as in exact arithmetic.)"""
    x = np.asarray(logits, F64)
    if not (t >= 0 and np.isfinite(t)) or np.isnan(x).any() or (x == np.inf).any() or (x == -np.inf).all():
        return None
    if t == 0:
        p = np.zeros(len(x))
        p[int(np.argmax(x))] = 1.0                                                  # the first of the largest
        return p
    with np.errstate(invalid="ignore"):
        return np.exp((x - x.max()) / t)


def distribution(logits, t):
    w = weights(logits, t)
    return None if w is None else w / w.sum()


def draw(p, u):
    """The first token whose running sum exceeds u times the total."""
    u = 0.0 if not u > 0 else min(u, 1 - 2.0 ** -24)
    run = np.cumsum(p)
    over = np.nonzero((run > u * run[-1]) & (p > 0))[0]
    return int(over[0]) if len(over) else int(np.nonzero(p > 0)[0][-1])


def parent_of(masks, j):
    return j - 1 if masks is None else (int(masks[j]) % (1 << 64) & ((1 << j) - 1)).bit_length() - 1


def accept(logits, ids, u, masks=None, draft=None, t=1.0):
    """One sequence's rows: (kept rows' numbers, the token after each, their log probabilities)."""
    n, t = len(ids), float(np.float32(t))
    path, tokens = [0], []
    if draft is None:
        while True:
            at = path[-1]
            p = weights(logits[at], t)
            tokens.append(-1 if p is None else draw(p, u[at]))
            kids = [j for j in range(at + 1, n) if ids[j] == tokens[-1] and tokens[-1] >= 0 and parent_of(masks, j) == at]
            if not kids:
                break
            path.append(kids[0])
    else:
        while True:
            at = path[-1]
            p = weights(logits[at], t)
            if p is None:
                tokens.append(-1)
                break
            if at + 1 == n:
                tokens.append(draw(p, u[0]))
                break
            x, q = int(ids[at + 1]), weights(draft[at + 1], t)
            q = None if q is None else q * (p.sum() / q.sum())                       # on p's scale
            inside = 0 <= x < len(p)
            uu = 0.0 if not u[at + 1] > 0 else min(u[at + 1], 1 - 2.0 ** -24)
            if t == 0:
                kept = inside and p[x] > 0
            else:
                kept = q is not None and inside and uu * q[x] < p[x]
            if kept:
                path.append(at + 1)
                tokens.append(x)
                continue
            rest = p if q is None or t == 0 else np.maximum(p - q, 0)
            tokens.append(draw(rest if rest.sum() > 0 else p, u[0]))
            break
    lp = []
    for j, x in zip(path, tokens):
        p = distribution(logits[j], t)
        if p is None:
            lp.append(np.nan)
        elif t == 0:
            lp.append(0.0)
        else:
            z = np.asarray(logits[j], F64) / t
            lp.append(z[x] - z.max() - np.log(np.exp(z - z.max()).sum()))
    return path, tokens, lp


# ----------------------------------------------------------------------------- pages
class Pool:
    """Tables and counts of a pool; copies [(from, to)] are what the calls move."""

    def __init__(self, refs, tables):
        self.refs, self.tables = np.array(refs, np.int64), np.array(tables, np.int64)

    def _named(self, block):
        return 0 <= block < len(self.refs)

    def _free(self):
        return [b for b in range(len(self.refs)) if self.refs[b] <= 0]

    def extend(self, tokens):
        free, asked, done, width = self._free(), 0, [], self.tables.shape[1]
        for b, n in enumerate(tokens):
            blocks = -(-max(0, int(n)) // PAGE)
            if blocks > width:
                done.append(0)
                continue
            miss = [e for e in range(blocks) if not self._named(self.tables[b, e])]
            first, asked = asked, asked + len(miss)
            ok = not miss or asked <= len(free)
            done.append(int(ok))
            if ok:
                for i, e in enumerate(miss):
                    self.tables[b, e] = free[first + i]
                    self.refs[free[first + i]] = 1
        return done

    def fork(self, src, dst, tokens):
        batch, width = self.tables.shape
        free, asked, done, copies = self._free(), 0, [], []
        tables, refs = self.tables.copy(), self.refs.copy()
        inside = lambda r: 0 <= r < batch  # noqa: E731
        for i, (a, b, n) in enumerate(zip(src, dst, tokens)):
            blocks = -(-int(n) // PAGE)
            ok = inside(a) and inside(b) and 0 <= n and blocks <= width and b not in dst[:i] and b not in src
            ok = ok and all(self._named(x) for x in self.tables[a, :blocks])
            if ok and n % PAGE:
                asked += 1
                ok = asked <= len(free)
            done.append(int(ok))
            if not ok:
                continue
            full = int(n) // PAGE
            tables[b] = -1
            tables[b, :full] = self.tables[a, :full]
            np.add.at(refs, self.tables[a, :full], 1)
            if n % PAGE:
                to = free[asked - 1]
                tables[b, full] = to
                refs[to] = 1
                copies.append((int(self.tables[a, full]), to))
        self.tables, self.refs = tables, refs
        return done, copies

    def free(self, seqs, tokens=None):
        """With tokens: which requests are served; one whose page kept in part others name too (before the call) is not."""
        keeps = [0] * len(seqs) if tokens is None else [max(0, int(n)) for n in tokens]
        done = [int(0 <= row < len(self.tables)) for row in seqs]
        for i, (row, n) in enumerate(zip(seqs, keeps)):
            if done[i] and n % PAGE and n // PAGE < self.tables.shape[1]:
                block = self.tables[row, n // PAGE]
                done[i] = int(not self._named(block) or self.refs[block] <= 1)
        for row, n, ok in zip(seqs, keeps, done):
            for e in range(-(-n // PAGE), self.tables.shape[1]) if ok else ():
                if self._named(self.tables[row, e]):
                    self.refs[self.tables[row, e]] -= 1
                self.tables[row, e] = -1
        return done

    def compact(self):
        used = self.refs > 0
        live = int(used.sum())
        holes = [b for b in range(live) if not used[b]]
        movers = [b for b in range(live, len(used)) if used[b]]
        place = np.where(used, np.arange(len(used)), -1)
        place[movers] = holes
        refs = np.where(used, self.refs, 0)
        refs[holes], refs[movers] = self.refs[movers], 0
        named = (self.tables >= 0) & (self.tables < len(used))
        self.tables = np.where(named, place[np.where(named, self.tables, 0)], -1)
        self.refs = refs
        return live, list(zip(movers, holes))


# ----------------------------------------------------------------------------- adapters
def lora(x, a, b, scale):
    """(scale b (a x) of rows x, the size of its terms: scale sum |b| |a x|, scale sum |b| sum |a| |x|)."""
    x, a, b = (np.asarray(t, F64) for t in (x, a, b))
    h = x @ a.T
    return scale * (h @ b.T), abs(scale) * (np.abs(h) @ np.abs(b).T), abs(scale) * ((np.abs(x) @ np.abs(a).T) @ np.abs(b).T)
