"""The paged cache in plain 64-bit arithmetic: the e4m3 codec, pages and attention, for the tests."""
import math

import numpy as np
import torch

EMIN = -110


def e4m3_values():
    """Value of each of the 256 codes."""
    v = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = (8 + m) * 2.0 ** (e - 10) if e else m * 2.0 ** -9
        v[c] = math.nan if c & 127 == 127 else (-x if c & 128 else x)
    return v


VALUES = e4m3_values()


def quantise(x):
    """Codes and scale bytes of rows x [.., d] (float64 holding bf16 values)."""
    x = np.asarray(x, dtype=np.float64)
    flat = x.reshape(-1, x.shape[-1])
    codes, scale = np.zeros(flat.shape, np.uint8), np.zeros(len(flat), np.uint8)
    grid = VALUES[:127]                                   # the non-negative finite values, ascending with the code
    for i, row in enumerate(flat):
        if not np.isfinite(row).all():
            codes[i], scale[i] = 0x7F, 255
            continue
        a, e = np.abs(row).max(), 0
        if a > 0:
            e = EMIN
            while a > math.ldexp(448.0, e):
                e += 1
        y = np.abs(np.ldexp(row, -e))
        hi = np.searchsorted(grid, y).clip(0, 126)        # grid[hi - 1] < y <= grid[hi]
        lo = np.maximum(hi - 1, 0)
        up, down = grid[hi] - y, y - grid[lo]
        c = np.where(up < down, hi, np.where(up > down, lo, np.where(hi % 2 == 0, hi, lo)))
        if e == 120:                                      # 256 * 2^120 is more than bf16 holds
            c = np.minimum(c, 0x77)
        codes[i], scale[i] = c | np.where(np.signbit(row), 128, 0), e + 127
    return codes.reshape(x.shape), scale.reshape(x.shape[:-1])


def decode(codes, scale):
    s = np.where(scale == 255, np.nan, np.ldexp(1.0, scale.astype(np.int64) - 127))
    return VALUES[codes] * s[..., None]


class Case:
    """Sequences with random pages: seqs = [(new tokens, length), ..]; some pages belong to nobody."""

    def __init__(self, seqs, H, d, page, fmt, seed=0, spare=3, junk=None, extra_cols=0, keys=1.0):
        self.seqs, self.H, self.d, self.page, self.fmt = seqs, H, d, page, fmt
        g = np.random.default_rng(seed)
        self.rng = g
        need = [-(-L // page) for _, L in seqs]
        self.n_pages = sum(need) + spare
        order = g.permutation(self.n_pages)
        cols = max(1, max(need)) + extra_cols
        self.table = np.full((len(seqs), cols), -7, np.int32)      # entries of nothing are not read
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.row_start = np.concatenate([[0], np.cumsum([n for n, _ in seqs])]).astype(np.int32)
        self.len = np.array([L for _, L in seqs], np.int32)
        self.rows = int(self.row_start[-1])
        shape = (self.n_pages, H, page, d)
        self.k = bf16(g.standard_normal(shape) * keys)
        self.v = bf16(g.standard_normal(shape))
        if junk is not None:                                       # what lies in slots of no position
            used = np.zeros((self.n_pages, page), bool)
            for b, (_, L) in enumerate(seqs):
                for j in range(L):
                    used[self.table[b, j // page], j % page] = True
            for x in (self.k, self.v):
                x[np.broadcast_to(~used[:, None, :, None], shape)] = junk
        if fmt == "e4m3":
            (self.kc, self.ks), (self.vc, self.vs) = quantise(self.k), quantise(self.v)
            self.k, self.v = decode(self.kc, self.ks), decode(self.vc, self.vs)

    def positions(self, b, h, lo, hi):
        """Keys and values of positions [lo, hi)."""
        j = np.arange(lo, hi)
        p, s = self.table[b, j // self.page], j % self.page
        return self.k[p, h, s], self.v[p, h, s]

    def cache(self, dkv, device="cuda"):
        if self.fmt == "e4m3":
            f8 = lambda x: torch.from_numpy(x).to(device).view(torch.float8_e4m3fn)
            return dkv.PagedCache(self.H, self.d, self.page, self.n_pages, "e4m3", k=f8(self.kc), v=f8(self.vc),
                                  k_scale=torch.from_numpy(self.ks).to(device), v_scale=torch.from_numpy(self.vs).to(device))
        b = lambda x: torch.from_numpy(x).to(device, torch.bfloat16)
        return dkv.PagedCache(self.H, self.d, self.page, self.n_pages, "bf16", k=b(self.k), v=b(self.v))

    def device_seqs(self, dkv, device="cuda"):
        t = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(device)
        return dkv.CacheSeqs(t(self.table), t(self.len), t(self.row_start))


def bf16(x):
    """x rounded to bf16, as float64."""
    return torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16).double().numpy()


def ends(p, L, block):
    return L if block == 0 else min(L, (p // block + 1) * block)


def attend(case, Q, window=0, sinks=0, block=1, scale=None, heads=None, rows=None):
    """{(h, row): (O, tolerance)} of the packed queries Q [H_q][rows][d] (float64).

    The tolerance, for each element, counts what a kernel may round (u = 2^-8, half a bf16 step):
    every weight to bf16, |dO| <= u sum w |v|; the output, u |O|; and in 32 bits a score's d products
    and sums, at most d 2^-23 sum |q k| each (a tensor core may cut instead of rounding), which moves
    every weight by that much relative and the sum by as much again, plus 2^-20 for the exponential
    and the sums of weights and of values."""
    Hq, _, d = Q.shape
    G = Hq // case.H
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out = {}
    for b, (n, L) in enumerate(case.seqs):
        for i in range(n):
            row = int(case.row_start[b]) + i
            if rows is not None and row not in rows:
                continue
            p = L - n + i
            end = ends(p, L, block) if p >= 0 else 0
            j = np.arange(end)
            if window:
                j = j[(j >= end - window) | (j < sinks)]
            for h in heads if heads is not None else range(Hq):
                if not len(j):
                    out[h, row] = np.zeros(d), np.zeros(d)
                    continue
                K, V = case.positions(b, h // G, 0, end)
                K, V = K[j], V[j]
                s = K @ Q[h, row] * scale
                with np.errstate(invalid="ignore", over="ignore"):
                    w = np.exp(s - s.max())
                    w = w / w.sum()
                    o = w @ V
                    wild = float((np.abs(K) @ np.abs(Q[h, row])).max()) * scale * d * 2.0 ** -23
                    tol = (w @ np.abs(V)) * (2.0 ** -8 + 2.0 * wild + 2.0 ** -20) * 1.01 + 2.0 ** -8 * np.abs(o) + 1e-30
                out[h, row] = o, tol
    return out


def check(O, ref):
    """O (a tensor [H_q][rows][d]) against attend()'s answer."""
    x = O.double().cpu().numpy()
    for (h, row), (o, tol) in ref.items():
        got = x[h, row]
        fine = np.isfinite(o)
        assert np.array_equal(np.isnan(got), np.isnan(o)) and np.array_equal(got[~fine & ~np.isnan(o)], o[~fine & ~np.isnan(o)]), (h, row)
        off = np.abs(got[fine] - o[fine]) - tol[fine]
        assert not fine.any() or off.max() <= 0, (h, row, float(off.max()), float(np.abs(got - o)[fine].max()))
