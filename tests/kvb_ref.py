"""The paged 8-bit cache and the page operators in plain numpy, written from the definitions in include/aasd.h: codes by
search among the values that they stand for, books as lists."""
from __future__ import annotations

import numpy as np

PAGE = 64
NONE = -1
LEAST = -64


def _values():
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    x = np.where(e > 0, (1 + m / 8.0) * 2.0 ** (e - 7.0), m * 2.0 ** -9)
    x = np.where(c >= 128, -x, x)
    x[[127, 255]] = np.nan
    return x


VALUES = _values()
_POS = VALUES[:127]                                  # ascending: 0 .. 448
_MID = (_POS[1:] + _POS[:-1]) / 2


def encode(x):
    """Nearest codes of float64 values up to 448 in size; between two, the even one."""
    a = np.abs(np.asarray(x, np.float64))
    low = np.searchsorted(_MID, a, side="left")      # (a on a midpoint: the code below it)
    tie = (low < 126) & (a == _MID[np.minimum(low, 125)])
    c = low + (tie & (low % 2 == 1))
    return np.where(np.signbit(x), c | 128, c).astype(np.uint8)


def fit(top):
    """Least exponent e >= -64 with top <= 448 * 2^e."""
    e = LEAST
    while top > 448.0 * 2.0 ** e:
        e += 1
    return e


def head_bytes(D):
    return 2 * PAGE * D + 16


def places(D, t):
    """Bytes of token t's channels inside the keys or the values."""
    ch = np.arange(D)
    row = min(D, 128)
    turn = t % 8 if row == 128 else t // 2 % 4
    return ch // row * (PAGE * row) + t * row + ((ch % row // 16) ^ turn) * 16 + ch % 16


class Block:
    """One half of one head's block of a page, seen in its bytes."""

    def __init__(self, raw, half, D):
        self.codes = raw[half * PAGE * D:(half + 1) * PAGE * D]
        self.word = raw[2 * PAGE * D + 4 * half:2 * PAGE * D + 4 * half + 4]
        self.D = D

    @property
    def e(self):
        return int(np.log2(float(np.ascontiguousarray(self.word).view("<f4")[0])))

    @e.setter
    def e(self, e):
        self.word[:] = np.array([2.0 ** e], "<f4").view(np.uint8)

    def value(self, t):
        return VALUES[self.codes[places(self.D, t)]] * 2.0 ** self.e

    def put(self, t, x):
        self.codes[places(self.D, t)] = encode(np.asarray(x, np.float64) * 2.0 ** -self.e)

    def grow(self, e, live):
        """Scale e; the live places follow."""
        old = [(t, self.value(t)) for t in live] if e > self.e else []
        self.e = e
        for t, x in old:
            self.put(t, x)


def write(raw, table, cached, kv_len, offs, k, v, D, placed=None):
    """k, v [T, Hkv, D] as they are to be stored (float32; rows that are not finite become zeros; rows where `placed` is
    false too).  Changes raw [pages, Hkv, bytes]."""
    for b in range(len(cached)):
        n = kv_len[b] - cached[b]
        for pg in range(cached[b] // PAGE, -(-kv_len[b] // PAGE) if n > 0 else 0):
            lo, hi = max(cached[b], pg * PAGE), min(kv_len[b], (pg + 1) * PAGE)
            for h in range(k.shape[1]):
                for half, x in enumerate((k, v)):
                    rows = []
                    for c in range(lo, hi):
                        t = offs[b] + c - cached[b]
                        r = np.asarray(x[t, h], np.float64)
                        rows.append(r if np.isfinite(r).all() and (placed is None or placed[t]) else np.zeros(D))
                    blk = Block(raw[table[b][pg], h], half, D)
                    older = range(cached[b] % PAGE) if pg * PAGE < cached[b] else range(0)
                    e = fit(max(np.abs(r).max() for r in rows))
                    if len(older):
                        blk.grow(max(e, blk.e), older)
                    else:
                        blk.e = e
                    for c, r in zip(range(lo, hi), rows):
                        blk.put(c % PAGE, r)


def load(raw, slot, D):
    """float64 keys and values [Hkv, D] at a slot."""
    return [np.stack([Block(raw[slot // PAGE, h], half, D).value(slot % PAGE) for h in range(raw.shape[1])]) for half in range(2)]


def path_of(node, parent):
    out = []
    while node >= 0:
        out.append(int(node))
        node = parent[node]
    return out[::-1]


def commit(raw, table, cached, path, D):
    """Moves one sequence's path in one layer [pages, Hkv, bytes]."""
    for h in range(raw.shape[1]):
        for half in range(2):
            place = lambda c: Block(raw[table[c // PAGE], h], half, D)                              # noqa: E731
            value = {cached + x: place(cached + x).value((cached + x) % PAGE) for x in path}
            scale = {pg: Block(raw[table[pg], h], half, D).e for pg in {(cached + x) // PAGE for x in path}}
            for pg in range(cached // PAGE, (cached + len(path) - 1) // PAGE + 1):
                new = {cached + i: cached + x for i, x in enumerate(path) if i != x and (cached + i) // PAGE == pg}
                if not new:
                    continue
                blk = Block(raw[table[pg], h], half, D)
                stay = [c % PAGE for c in range(pg * PAGE, min(new))]
                blk.grow(max([blk.e] + [scale[s // PAGE] for s in new.values()]), stay)
                for to, src in new.items():
                    blk.put(to % PAGE, value[src])


class Books:
    """Page tables, stack and holders as lists."""

    def __init__(self, table, held, stack, shares, cached, width):
        self.table, self.stack, self.shares, self.cached, self.width = [list(r) for r in table], list(stack), list(shares), list(cached), width
        assert [len(r) for r in self.table] == list(held)

    def free(self, keep, new=None):
        gone = []
        for b, n in enumerate(keep):
            if n == NONE:
                continue
            need = -(-(n + (new[b] if new is not None else 0)) // PAGE)
            while len(self.table[b]) > need:
                p = self.table[b].pop()
                self.shares[p] -= 1
                if self.shares[p] < 0:
                    self.shares[p] = 0
                    gone.append(p)
        self.stack += sorted(gone)

    def fork(self, src, dst, length=None):
        """Returns (new_len, copy_src, copy_dst) per fork, whether the stack ran out, whether something was refused."""
        B, out, full, bad = len(self.table), [], False, False
        was = [len(r) for r in self.table]
        taken, asked, start, claimed = set(), 0, len(self.stack), set(dst)
        for i, (s, d) in enumerate(zip(src, dst)):
            ok = 0 <= d < B and was[d] == 0 and d not in taken and 0 <= s < B and not (s in claimed and was[s] == 0)
            if 0 <= d < B and was[d] == 0:
                taken.add(d)
            n = 0
            if ok:
                n = self.cached[s] if length is None else length[i]
                ok = 0 <= n <= self.cached[s] and was[s] * PAGE >= n
            if not ok:
                bad = True
                out.append((NONE, NONE, NONE))
                continue
            if n % PAGE:
                asked += 1
                if asked > start:
                    full = True
                    out.append((NONE, NONE, NONE))
                    continue
            self.table[d] = self.table[s][:n // PAGE]
            for p in self.table[d]:
                self.shares[p] += 1
            self.cached[d] = n
            if n % PAGE:
                self.table[d].append(self.stack.pop())
                out.append((n, self.table[s][n // PAGE], self.table[d][-1]))
            else:
                out.append((n, NONE, NONE))
        return out, full, bad

    def compact(self):
        """Returns the new number of each page (NONE: free) and the moves (from, to)."""
        N = len(self.shares)
        used = N - len(self.stack)
        idle = set(self.stack)
        far = [p for p in range(used, N) if p not in idle]
        holes = [p for p in range(used) if p in idle]
        to = {p: p for p in range(N) if p not in idle}
        to.update(zip(far, holes))
        shares = [0] * N
        for p, q in to.items():
            shares[q] = self.shares[p]
        self.shares = shares
        self.table = [[to[p] for p in r] for r in self.table]
        self.stack = list(range(N - 1, used - 1, -1))
        return [to.get(p, NONE) for p in range(N)], list(zip(far, holes))
