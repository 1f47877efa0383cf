"""fp64 oracle of the operators around the paged 4-bit cache: the e2m1 / e4m3 number formats, the quantised entries, the norm and rotation of
queries and keys, and the bookkeeping of pages.

TEST INFRASTRUCTURE ONLY: imported by tests; never by the product path.  Plain Python and NumPy, float64, one row, token or page at a time.

  * e2m1 holds 0, .5, 1, 1.5, 2, 3, 4, 6 with a sign; e4m3 holds 448 at most, 2^-9 at least, and a NaN (0x7F, 0xFF).  Rounding: nearest,
    ties to the even code, beyond the largest the largest.
  * A block of 16 numbers: scale = e4m3(max|x| 2^-e / 6), codes = e2m1(x 2^-e / scale); scale 0: zeros; a NaN in the block: all NaN.
  * Attention over the cache is attn_oracle's attention over the values that the codes stand for.
  * Pages: a row's pages in order, a count per page, a list of free pages whose last entry is taken first; every call works through its list
    of rows one after another.

Pins: tests/test_oracle_kv4.py.
"""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])

SEQ_OK, SEQ_BAD_ROW, SEQ_BAD_CTX, SEQ_BAD_PAGE, SEQ_NO_PAGES = 0, 5, 7, 8, 9


def e4m3_value(byte: int) -> float:
    """What an e4m3 byte stands for."""
    s, e, m = byte >> 7, (byte >> 3) & 15, byte & 7
    if e == 15 and m == 7:
        return float("nan")
    v = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
    return -v if s else v


E4M3 = np.array([e4m3_value(b) for b in range(127)])         # 0 .. 448, ascending


def nearest(x: float, grid: np.ndarray) -> int:
    """Place in the ascending grid of the number nearest to x >= 0: ties to the even place, beyond the end the last."""
    if x >= grid[-1]:
        return len(grid) - 1
    d = np.abs(grid - x)
    best = np.flatnonzero(d == d.min())
    return int(best[0] if len(best) == 1 or best[0] % 2 == 0 else best[1])


def quantise_block(x, e: int):
    """16 numbers -> (codes [16], scale byte)."""
    x = np.asarray(x, np.float64)
    if np.isnan(x).any():
        return np.zeros(16, np.uint8), 0x7F
    y = np.clip(x * 2.0 ** -e, -1e30, 1e30)                  # infinities count as very large numbers
    sb = nearest(np.abs(y).max() / 6.0, E4M3)
    s = E4M3[sb]
    codes = np.zeros(16, np.uint8)
    for i in range(16):
        mag = nearest(abs(y[i]) / s, E2M1) if s > 0 else 0
        codes[i] = mag | (8 if y[i] < 0 else 0)
    return codes, sb


def block_values(codes, sb: int, e: int) -> np.ndarray:
    v = np.array([(-1.0 if c & 8 else 1.0) * E2M1[c & 7] for c in codes])
    with np.errstate(invalid="ignore"):
        return v * e4m3_value(int(sb)) * 2.0 ** e


def quantise(x, e: int = 0) -> np.ndarray:
    """x [..., 128] -> the values the cache stands for."""
    x = np.asarray(x, np.float64)
    rows = x.reshape(-1, 8, 16)
    out = np.empty_like(rows)
    for i in range(rows.shape[0]):
        for j in range(8):
            c, sb = quantise_block(rows[i, j], e)
            out[i, j] = block_values(c, sb, e)
    return out.reshape(x.shape)


def entry(pages, table, row, pos, head, which, page_size, e: int = 0) -> np.ndarray:
    """The 128 values held at a position: pages uint8 [n_pages, Hkv, 2, page_size * 72]."""
    raw = pages[table[row][pos // page_size], head, which]
    at = pos % page_size
    codes = raw[at * 64:at * 64 + 64]
    scales = raw[page_size * 64 + at * 8:page_size * 64 + at * 8 + 8]
    nib = np.empty(128, np.uint8)
    nib[0::2], nib[1::2] = codes & 15, codes >> 4
    return np.concatenate([block_values(nib[16 * j:16 * j + 16], scales[j], e) for j in range(8)])


def cache_values(pages, table, row, length, page_size, k_exp=0, v_exp=0):
    """Keys and values [length, Hkv, 128] of a row's first positions (``entry`` for all of them at once)."""
    pos = np.arange(length)
    raw = pages[np.asarray(table)[row][pos // page_size]]                               # [length, Hkv, 2, bytes]
    at = pos % page_size
    ci = at[:, None] * 64 + np.arange(64)
    si = page_size * 64 + at[:, None] * 8 + np.arange(8)
    codes = np.take_along_axis(raw, ci[:, None, None, :], axis=3)
    scales = np.take_along_axis(raw, si[:, None, None, :], axis=3)
    nib = np.stack([codes & 15, codes >> 4], axis=-1).reshape(*codes.shape[:3], 128)
    v = np.where(nib & 8, -1.0, 1.0) * E2M1[nib & 7]
    sc = np.array([e4m3_value(b) for b in range(256)])[scales]
    with np.errstate(invalid="ignore"):
        v = v * np.repeat(sc, 16, axis=-1)
    return v[:, :, 0] * 2.0 ** k_exp, v[:, :, 1] * 2.0 ** v_exp


# ---------------------------------------------------------------------------
def axis_of(n: int, sections=None, turns=False):
    """Axis of each of the n pairs."""
    if sections is None:
        return [0] * n
    if turns:
        return [j % 3 if j % 3 and j // 3 < sections[j % 3] else 0 for j in range(n)]
    return [0] * sections[0] + [1] * sections[1] + [2] * sections[2]


def norm_rope(x, pos, inv_freq, weight=None, offset=0.0, eps=1e-6, normalise=True, style="half", sections=None, turns=False, mscale=1.0):
    """x [T, H, dh]; pos [axes, T] integers; inv_freq [n] (any floating type, taken exactly)."""
    y = np.array(x, np.float64)
    T, H, dh = y.shape
    n = len(inv_freq)
    if normalise:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps)
        if weight is not None:
            y = y * (np.asarray(weight, np.float64) + offset)
    ax = axis_of(n, sections, turns)
    out = y.copy()
    for t in range(T):
        for j in range(n):
            a = float(pos[ax[j]][t]) * float(inv_freq[j])
            c, s = np.cos(a) * mscale, np.sin(a) * mscale
            i0, i1 = (j, j + n) if style == "half" else (2 * j, 2 * j + 1)
            out[t, :, i0] = y[t, :, i0] * c - y[t, :, i1] * s
            out[t, :, i1] = y[t, :, i0] * s + y[t, :, i1] * c
    return out


# ---------------------------------------------------------------------------
class Pages:
    """The page table as lists.  Pools: arrays [n_pages, ...]."""

    def __init__(self, n_rows, max_pages, n_pages, page_size, pools=()):
        self.max_pages, self.n_pages, self.P = max_pages, n_pages, page_size
        self.rows = [[] for _ in range(n_rows)]
        self.free = list(range(n_pages - 1, -1, -1))
        self.pools = [np.array(p) for p in pools]

    def refs(self):
        r = [0] * self.n_pages
        for row in self.rows:
            for p in row:
                r[p] += 1
        return r

    def table(self):
        return [row + [-1] * (self.max_pages - len(row)) for row in self.rows]

    def _listed(self, rows):
        """(index, row) of the entries that count, and the status words."""
        st, seen, use = [SEQ_OK] * len(rows), set(), []
        for i, r in enumerate(rows):
            if r == -1:
                continue
            if r < 0 or r >= len(self.rows) or r in seen:
                st[i] = SEQ_BAD_ROW
            else:
                use.append((i, r))
            seen.add(r)
        return use, st

    def fork(self, src, dst):
        st = [SEQ_OK] * len(src)
        before = [list(r) for r in self.rows]
        for i, (s, d) in enumerate(zip(src, dst)):
            if s == -1 or d == -1:
                continue
            live = [(t, e) for t, e in zip(src, dst) if t != -1 and e != -1]                # (a pair that is passed over names nothing)
            named = [e for t, e in zip(src[:i], dst[:i]) if t != -1]
            ok = 0 <= s < len(self.rows) and 0 <= d < len(self.rows) and d not in named and all(t != d for t, _ in live)
            if not ok or before[d]:
                st[i] = SEQ_BAD_ROW
                continue
            self.rows[d] = list(before[s])
        return st

    def reserve(self, rows, start, end):
        use, st = self._listed(rows)
        work = []
        for i, r in use:
            if start[i] < 0 or end[i] < start[i] or -(-end[i] // self.P) > self.max_pages:
                st[i] = SEQ_BAD_CTX
            else:
                work.append((i, r))
        refs, table, free, moves = self.refs(), [list(r) for r in self.rows], list(self.free), []
        lack = False
        for i, r in work:
            have, need = len(table[r]), -(-end[i] // self.P)
            if end[i] > start[i]:
                for k in range(start[i] // self.P, min(have, need)):
                    p = table[r][k]
                    if refs[p] > 1:
                        if not free:
                            lack = True
                            break
                        new = free.pop()
                        moves.append((p, new))
                        refs[p] -= 1
                        refs[new] = 1
                        table[r][k] = new
            while not lack and len(table[r]) < need:
                if not free:
                    lack = True
                    break
                table[r].append(free.pop())
                refs[table[r][-1]] = 1
            if lack:
                break
        if lack:
            for i, _ in work:
                st[i] = SEQ_NO_PAGES
            return st
        self.rows, self.free = table, free
        for pool in self.pools:
            old = pool.copy()
            for s, d in moves:
                pool[d] = old[s]
        return st

    def release(self, rows, keep):
        use, st = self._listed(rows)
        refs, order, gone = self.refs(), [], []
        for i, r in use:
            if keep[i] < 0:
                st[i] = SEQ_BAD_CTX
                continue
            left = min(len(self.rows[r]), -(-keep[i] // self.P))
            gone += self.rows[r][left:]
            self.rows[r] = self.rows[r][:left]
        for p in gone:
            refs[p] -= 1
        for p in gone:
            if refs[p] == 0 and p not in order:
                order.append(p)
        self.free += order[::-1]
        return st

    def compact(self):
        refs = self.refs()
        live = sum(1 for r in refs if r)
        movers = [p for p in range(live, self.n_pages) if refs[p]]
        holes = [p for p in range(live) if not refs[p]]
        to = dict(zip(movers, holes))
        self.rows = [[to.get(p, p) for p in row] for row in self.rows]
        for pool in self.pools:
            for s, d in to.items():
                pool[d] = pool[s]
        self.free = list(range(self.n_pages - 1, live - 1, -1))
        return to
