"""Norm and rotation, pages of several sequences, and chosen pages in plain 64-bit arithmetic, for the tests."""
import math

import numpy as np

import cache_ref

SMIN, WILD = -50, 2.0 ** 40


# ---------------------------------------------------------------- norm and rotation
def norm_rope(x, coord, theta, pairs, half, norm, eps, weight):
    """Rows x [heads][rows][d] (float64) and, for each element, how far fp32 may be from that before the output's rounding.

    The relative error of a normed value is at most (d / 2 + 8) 2^-24: half of that of a sum of d squares (each of d
    products and sums rounds once), the reciprocal root's 2 ulp and its argument's product and sum, and the products with
    the root and the weight.  An angle is off by 2^-22 + |a| 2^-51, its sine and cosine by two steps of 2^-24 more, and
    the two products and the sum of a rotation round three times."""
    d = x.shape[-1]
    x = np.asarray(x, np.float64)
    if norm:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1.0 if weight is None else weight)
    axis = np.repeat(np.arange(len(pairs)), pairs)
    a = coord[axis].T.astype(np.float64) * theta                      # [rows][d / 2]
    p, q = (x[..., :d // 2], x[..., d // 2:]) if half else (x[..., 0::2], x[..., 1::2])
    y0, y1 = p * np.cos(a) - q * np.sin(a), p * np.sin(a) + q * np.cos(a)
    step = (np.abs(p) + np.abs(q)) * ((d / 2 + 8 if norm else 0) * 2.0 ** -24 + 5 * 2.0 ** -24 + 2.0 ** -22 + np.abs(a) * 2.0 ** -51)
    join = (lambda u, v: np.concatenate([u, v], -1)) if half else (lambda u, v: np.stack([u, v], -1).reshape(*u.shape[:-1], d))
    return join(y0, y1), join(step, step)


def check_rows(got, want, step):
    """bf16 rows against norm_rope's answer: `step` and half a step of bf16 (2^-8 of the value)."""
    got = got.double().cpu().numpy()
    off = np.abs(got - want) - (step * 1.01 + (np.abs(want) + step) * 2.0 ** -8 + 2.0 ** -134)
    assert np.isfinite(got).all() and off.max() <= 0, float(off.max())


# ---------------------------------------------------------------- pages
class Book:
    """Tables, lengths, counts and pool rows, one sequence after the other.  rows: arrays [n_pages][H][page_len][..]."""

    def __init__(self, n_pages, page, rows):
        self.page, self.refs, self.rows = page, [0] * n_pages, [r.copy() for r in rows]
        self.table, self.length = [], []

    def free(self):
        return [p for p, r in enumerate(self.refs) if r == 0]

    def fork(self, parents):
        old = self.table
        for row in old:
            for p in row:
                if p >= 0:
                    self.refs[p] -= 1
        self.length = [self.length[a] if a >= 0 else 0 for a in parents]
        self.table = [list(old[a]) if a >= 0 else [] for a in parents]
        for row in self.table:
            for p in row:
                if p >= 0:
                    self.refs[p] += 1

    def extend(self, add):
        """False: too few pages, nothing done."""
        save = [list(r) for r in self.table], list(self.length), list(self.refs), [r.copy() for r in self.rows]
        free = self.free()                                            # (pages given up by this call are not given out by it)
        for b, more in enumerate(add):
            row, n = self.table[b], self.length[b]
            if more and n % self.page and self.refs[row[n // self.page]] > 1:
                if not free:
                    break
                src, dst = row[n // self.page], free.pop(0)
                self.refs[src] -= 1
                self.refs[dst] = 1
                row[n // self.page] = dst
                for r in self.rows:
                    r[dst, :, :n % self.page] = r[src, :, :n % self.page]
            while len(row) * self.page < n + more and free:
                row.append(free.pop(0))
                self.refs[row[-1]] = 1
            if len(row) * self.page < n + more:
                break
            self.length[b] = n + more
        else:
            return True
        self.table, self.length, self.refs, self.rows = save
        return False

    def release(self, first, last):
        for b, (lo, hi) in enumerate(zip(first, last)):
            n, lo = self.length[b], max(lo, 0)
            for k, p in enumerate(self.table[b]):
                a, z = k * self.page, min(n, (k + 1) * self.page)
                if p >= 0 and lo <= a < n and z <= hi:
                    self.refs[p] -= 1
                    self.table[b][k] = -1
            if hi >= n and lo < n and hi > lo:
                self.length[b] = lo
                self.table[b] = self.table[b][:-(-lo // self.page)]

    def compact(self, keep):
        free, tables, gone, old_rows = self.free(), [], [], [r.copy() for r in self.rows]
        for b, mine in enumerate(keep):
            old, row, same = self.table[b], [], True
            for k in range(0, len(mine), self.page):
                part = mine[k:k + self.page]
                same = same and list(part) == list(range(k, k + len(part)))
                if same:
                    row.append(old[k // self.page])
                    continue
                row.append(free.pop(0))
                self.refs[row[-1]] = 1
                for i, j in enumerate(part):
                    for r, o in zip(self.rows, old_rows):
                        r[row[-1], :, i] = o[old[j // self.page], :, j % self.page]
            gone += [p for k, p in enumerate(old) if p >= 0 and not (k < len(row) and row[k] == p)]
            tables.append(row)
        for p in gone:
            self.refs[p] -= 1
        self.table, self.length = tables, [len(m) for m in keep]

    def padded(self, cols):
        return np.array([r + [-1] * (cols - len(r)) for r in self.table], np.int32).reshape(len(self.table), cols)


# ---------------------------------------------------------------- chosen pages
def codes8(x):
    """(codes, exponent) of one row, or (zeros, None) where it has none."""
    a = np.abs(x).max()
    if not a < WILD:
        return np.zeros(len(x)), None
    e = SMIN
    while a > 127 * 2.0 ** e:
        e += 1
    return np.rint(np.ldexp(x, -e)), e


def summaries(case, pages=None, code=None, scale=None):
    """code [n_pages][H][d], scale [n_pages][H] of the pages {(sequence, entry)} (None: all held)."""
    code = np.zeros((case.n_pages, case.H, case.d), np.int8) if code is None else code
    scale = np.full((case.n_pages, case.H), 77, np.uint8) if scale is None else scale
    for b, (_, L) in enumerate(case.seqs):
        for k in range(-(-L // case.page)):
            if pages is not None and (b, k) not in pages:
                continue
            p, m = case.table[b, k], min(case.page, L - k * case.page)
            for h in range(case.H):
                with np.errstate(invalid="ignore"):
                    c, e = codes8(math_mean(case.k[p, h, :m]))
                code[p, h], scale[p, h] = c, 255 if e is None else e + 127
    return code, scale


def math_mean(rows):
    """The columns' sums exactly rounded, then divided."""
    if not np.isfinite(rows).all():
        return np.full(rows.shape[1], np.nan)
    return np.array([math.fsum(col) for col in rows.T]) / len(rows)


def tiles(case, tile):
    for b, (n, L) in enumerate(case.seqs):
        for i in range(0, n, tile):
            yield b, i, min(tile, n - i), int(case.row_start[b]) // tile + b + i // tile


def choose(case, Q, code, scale, top, tile, block, sinks, local, width):
    """Lists [H][slots][width] of the queries Q [H_q][rows][d] (float64)."""
    G, H = Q.shape[0] // case.H, case.H
    out = np.full((H, case.rows // tile + len(case.seqs), width), -1, np.int32)
    for b, i, m, slot in tiles(case, tile):
        n, L = case.seqs[b]
        p1 = L - n + i + m - 1
        if p1 < 0:
            continue
        p0 = max(L - n + i, 0)
        end = cache_ref.ends(p0, L, block)
        whole = [k for k in range(-(-L // case.page)) if min(L, (k + 1) * case.page) <= end]
        forced = set(range(max(0, p0 // case.page - (local - 1)), p1 // case.page + 1)) | {k for k in whole if k < sinks}
        for h in range(H):
            best = {k: -math.inf for k in whole if k not in forced}
            for r in range(int(case.row_start[b]) + i, int(case.row_start[b]) + i + m):
                for g in range(G):
                    c, e = codes8(Q[h * G + g, r])
                    if e is None:
                        continue
                    for k in best:
                        p = case.table[b, k]
                        if scale[p, h] != 255:
                            best[k] = max(best[k], math.ldexp(float(c @ code[p, h].astype(np.float64)), e + int(scale[p, h]) - 127))
            rest = sorted((-v, k) for k, v in best.items() if v > -math.inf)[:top]
            row = sorted(forced | {k for _, k in rest})
            out[h, slot, :len(row)] = row
    return out


def attend(case, Q, lists, tile, block=1, scale=None, hidden=()):
    """{(h, row): (O, tolerance)}, the tolerance as cache_ref.attend derives it.  hidden: positions left out."""
    G, d = Q.shape[0] // case.H, case.d
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out = {}
    for b, i, m, slot in tiles(case, tile):
        n, L = case.seqs[b]
        for h in range(Q.shape[0]):
            line = [int(k) for k in lists[h // G, slot]]
            line = line[:line.index(-1)] if -1 in line else line
            pos = np.array([k * case.page + x for k in line for x in range(case.page)], np.int64)
            for row in range(int(case.row_start[b]) + i, int(case.row_start[b]) + i + m):
                p = L - n + row - int(case.row_start[b])
                j = pos[pos < (cache_ref.ends(p, L, block) if p >= 0 else 0)]
                j = j[~np.isin(j, list(hidden))]
                if not len(j):
                    out[h, row] = np.zeros(d), np.zeros(d)
                    continue
                at, s = case.table[b, j // case.page], j % case.page
                K, V = case.k[at, h // G, s], case.v[at, h // G, s]
                x = K @ Q[h, row] * scale
                with np.errstate(invalid="ignore", over="ignore"):
                    if (x == -math.inf).all():
                        out[h, row] = np.zeros(d), np.zeros(d)
                        continue
                    w = np.exp(x - x.max())
                    w = w / w.sum()
                    o = w @ V
                    wild = float((np.abs(K) @ np.abs(Q[h, row])).max()) * scale * d * 2.0 ** -23
                    tol = (w @ np.abs(V)) * (2.0 ** -8 + 2.0 * wild + 2.0 ** -20) * 1.01 + 2.0 ** -8 * np.abs(o) + 1e-30
                out[h, row] = o, tol
    return out
