"""What a server does around the paged cache of the window, as cases to time and compare.

  rope     dkv_norm_rope, dkv_cache_write_norm_rope: queries and keys of every head normed and rotated to their
           positions in one pass, dense or with the keys and values put into their pages;
  fork     dkv_cache_fork, dkv_cache_extend: sequences go on as their parents' tables say (shared pages, counted), then
           grow: fresh pages, and a copy of a shared last page;
  compact  dkv_cache_compact: the kept positions of every sequence moved up to its front;
  choose   dkv_cache_summarise, dkv_cache_choose: an 8-bit mean key of the pages that new tokens lie on, and for each
           tile of tokens and key head the pages whose summaries score best;
  chosen   dkv_cache_attend_chosen: attention of each tile over its listed pages.

Sequence b holds L tokens; its n newest are rows [row_start[b], row_start[b + 1]) of the packed tensors
[heads][rows][d], at positions L - n .. L - 1.  Position j is slot j % page_len of page table[b][j / page_len]; a page
is [heads][page_len][d].  Tile t of a sequence (tokens [t tile, (t + 1) tile) of its new ones) has slot
row_start[b] / tile + b + t of the lists.
"""
import math
import random

import torch

own = False

EMIN = -110                      # smallest exponent of an e4m3 row's scale
SMIN, WILD = -50, 2.0 ** 40      # of a summary's; magnitudes that it does not hold

_BASE = dict(kind="rope", fmt="bf16", d=128, page=64, Hq=12, Hkv=12, B=1, n_lo=1, n_hi=1, past_lo=0, past_hi=0, mix=0,
             dense=False, axes=1, half=False, norm=True, B2=1, keep="window", window=0, sinks=0, block=1, tile=1, sink_pages=1,
             local_pages=2, top=16)


def _case(**kw):
    c = dict(_BASE)
    c.update(kw)
    return c


def listed():
    return [
        # One new token each of 32 sequences of text, grouped heads, into a quantised cache: a server's step, launches count.
        _case(name="rope_token", fmt="e4m3", Hq=40, Hkv=8, B=32, past_lo=700, past_hi=9360, mix=1),
        # A frame and a token of a small model, far on in its text; dense, for the bank.
        _case(name="rope_frame_d64", d=64, Hq=24, Hkv=8, n_lo=1561, n_hi=1561, past_lo=1000000, past_hi=1000000, dense=True,
              half=True),
        # A 3-frame block of a layer of 40 heads, rotated by time, row and column, into its pages.
        _case(name="rope_block", page=128, Hq=40, Hkv=40, n_lo=4680, n_hi=4680, past_lo=9360, past_hi=9360, axes=3),
        # A step of 48 parallel continuations: some go on twice, some end, all get a few tokens' room.
        _case(name="fork_token", kind="fork", Hkv=8, B=48, B2=48, n_lo=1, n_hi=5, past_lo=90, past_hi=2000, mix=2),
        # Three prompts, each the start of many continuations on large pages of a layer of 40 heads.
        _case(name="fork_prompt", kind="fork", page=256, Hkv=40, B=3, B2=64, n_lo=1, n_hi=1, past_lo=2600, past_hi=4800,
              mix=3),
        # The sink frame and the window of a long video moved together, quantised, at an odd offset.
        _case(name="compact_window", kind="compact", fmt="e4m3", Hkv=40, B=2, past_lo=14045, past_hi=16011, window=7800,
              sinks=1560, mix=4),
        # Prompts thinned out: three positions of five stay, small pages.
        _case(name="compact_thin", kind="compact", page=16, Hkv=8, B=8, past_lo=300, past_hi=4000, keep="thin", mix=5),
        # One token each of 32 long sequences, grouped heads: 16 pages of up to 469 each.
        _case(name="choose_token", kind="choose", Hq=40, Hkv=8, B=32, past_lo=700, past_hi=30000, mix=6),
        # A block's queries in tiles of a page, over 30 frames: 48 pages of 732.
        _case(name="choose_block", kind="choose", n_lo=4680, n_hi=4680, past_lo=42120, past_hi=42120, block=4680, tile=64,
              top=48),
        # The attention of those 32 tokens over 32 pages each, quantised.
        _case(name="chosen_token", kind="chosen", fmt="e4m3", Hq=40, Hkv=8, B=32, past_lo=2100, past_hi=30000, top=29, mix=7),
        # Chunks of a small model's prompts, four sequences, each tile of 16 tokens over its own pages of 16.
        _case(name="chosen_chunk_d64", kind="chosen", d=64, page=16, Hq=24, Hkv=8, B=4, n_lo=333, n_hi=700, past_lo=0,
              past_hi=7600, tile=16, top=40, mix=8),
        # A block of a layer of 40 heads over 30 frames: a tile of 128 sees 28 pages of 128.
        _case(name="chosen_block", kind="chosen", page=128, Hq=40, Hkv=40, n_lo=4680, n_hi=4680, past_lo=42120, past_hi=42120,
              block=4680, tile=128, top=24),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    top = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["rope", "rope", "fork", "compact", "choose", "chosen", "chosen"])
        c = _case(kind=kind, fmt=rng.choice(["bf16", "e4m3"]), d=rng.choice([128, 128, 64]),
                  page=rng.choice([16, 32, 64, 128, 256]), B=_log(rng, 1, 48), mix=rng.randrange(1 << 20))
        hkv = rng.choice([1, 2, 4, 8, 12, 40])
        group = rng.choice([1, 1, 2, 3, 4, 5, 7, 8]) if kind in ("rope", "choose", "chosen") else 1
        c["Hkv"], c["Hq"] = hkv, hkv * group
        chunk = 1 if rng.random() < 0.35 else _log(rng, 2, 4680)
        c["past_hi"] = _log(rng, 16, 131000) if chunk == 1 else _log(rng, 16, 42120)
        if kind == "rope":
            c["dense"] = rng.random() < 0.3
            c["axes"], c["half"], c["norm"] = rng.choice([1, 3]), rng.random() < 0.5, rng.random() < 0.8
            if c["fmt"] == "e4m3":       # (a scale byte is a whole number, and one in many millions lies on a border)
                chunk = min(chunk, 200)
        elif kind == "fork":
            chunk = _log(rng, 1, 300)
            c["B2"] = _log(rng, 1, 64)
            c["past_hi"] = _log(rng, 16, 9360)
        elif kind == "compact":
            chunk = 0
            c["keep"] = rng.choice(["window", "thin", "any"])
            c["past_hi"] = _log(rng, 16, 16000)
            c["window"], c["sinks"] = _log(rng, 16, 8000), rng.choice([0, 4, _log(rng, 1, 1560)])
        else:
            c["block"] = rng.choice([1, 1, 0, chunk])
            c["tile"] = 1 if chunk == 1 else rng.choice([1, 8, 16, 64, 128])
            c["sink_pages"], c["local_pages"], c["top"] = rng.choice([0, 1, 2]), rng.choice([1, 2, 3]), _log(rng, 1, 60)
        c["n_hi"] = chunk
        c["n_lo"] = rng.choice([chunk, -(-chunk // 3)])
        c["past_lo"] = rng.choice([c["past_hi"], c["past_hi"] // 8, 0])
        total = (c["B"] + (c["B2"] if kind == "fork" else 0)) * (c["past_hi"] + chunk + c["page"])
        if total * hkv * c["d"] * 4 > 3e9 or c["B"] * chunk * c["Hq"] * c["d"] > 2e8 or _cost(c) > top:
            continue
        if kind == "choose" and c["B"] * chunk * c["Hq"] * (c["past_hi"] + chunk) / c["page"] > 2e9:
            continue
        if kind == "chosen":
            pairs = c["B"] * -(-chunk // c["tile"]) * hkv * _width(c) * c["page"]      # keys that the tiles list
            if pairs * c["d"] > 2e10 or pairs * min(chunk, c["tile"]) * group > 1e10:
                continue
        return c


# ---------------------------------------------------------------- sizes and work
def _sizes(c):
    """(new tokens, length) of each sequence."""
    r = random.Random(c["mix"] * 1000003 + c["B"])
    out = []
    for _ in range(c["B"]):
        n = r.randint(c["n_lo"], c["n_hi"])
        out.append((n, n + r.randint(c["past_lo"], c["past_hi"])))
    return out


def _parents(c):
    """Parent of each continuation (-1: none) and the tokens that it gets room for."""
    r = random.Random(c["mix"] * 1000033 + c["B2"])
    return ([r.randrange(c["B"]) if r.random() < 0.95 else -1 for _ in range(c["B2"])],
            [r.randint(c["n_lo"], c["n_hi"]) for _ in range(c["B2"])])


def _kept(c):
    """Kept positions of each sequence, in their new order."""
    r = random.Random(c["mix"] * 1000037 + c["B"])
    out = []
    for _, length in _sizes(c):
        if c["keep"] == "window":
            out.append(sorted(set(range(min(length, c["sinks"]))) | set(range(max(0, length - c["window"]), length))))
        elif c["keep"] == "thin":
            out.append([j for j in range(length) if r.random() < 0.6])
        else:
            out.append([r.randrange(length) for _ in range(r.randint(0, length))] if length else [])
    return out


def _width(c):
    return c["sink_pages"] + c["local_pages"] + (c["tile"] + c["page"] - 2) // c["page"] + c["top"]


def _end(c, p, length):
    return length if c["block"] == 0 else min(length, (p // c["block"] + 1) * c["block"])


def _tiles(c):
    """(sequence, first token, tokens, slot, first page of the local ones, pages that end before the first token's view,
    last page of the tile's own) of every tile, and the number of slots."""
    out, row = [], 0
    for b, (n, length) in enumerate(_sizes(c)):
        for i in range(0, n, c["tile"]):
            m = min(c["tile"], n - i)
            p0, p1 = length - n + i, length - n + i + m - 1
            e = _end(c, p0, length)
            whole = -(-length // c["page"]) if e == length else e // c["page"]
            out.append((b, i, m, row // c["tile"] + b + i // c["tile"], max(0, p0 // c["page"] - (c["local_pages"] - 1)), whole,
                        p1 // c["page"]))
        row += n
    return out, row // c["tile"] + c["B"]


def work(c):
    d = c["d"]
    row = 4 * d if c["fmt"] == "bf16" else 2 * d + 2          # a position's key and value of a head in the cache
    rows = sum(n for n, _ in _sizes(c))
    if c["kind"] == "rope":
        out = 4 * d if c["dense"] else 4 * d + row            # keys in and out, or keys and values in, pages out
        return {"bytes": rows * (4 * d * c["Hq"] + out * c["Hkv"]),
                "flops": rows * (c["Hq"] + c["Hkv"]) * d * (7 if c["norm"] else 3)}
    if c["kind"] == "fork":
        sizes, page = _sizes(c), c["page"]
        parents, _ = _parents(c)
        part = [sizes[p][1] % page for p in parents if p >= 0]
        once = [sizes[p][1] % page for p in set(parents) - {-1}]
        tables = sum(-(-sizes[p][1] // page) for p in parents if p >= 0)
        return {"bytes": 2 * (sum(part) - sum(once)) * c["Hkv"] * row + 8 * tables, "flops": 0}
    if c["kind"] == "compact":
        moved = 0
        for kept in _kept(c):
            same = next((i for i, j in enumerate(kept) if i != j), len(kept))
            moved += len(kept) - (same if same == len(kept) else same // c["page"] * c["page"])
        return {"bytes": 2 * moved * c["Hkv"] * row + 4 * sum(len(k) for k in _kept(c)), "flops": 0}
    tiles, slots = _tiles(c)
    lists = 4 * c["Hkv"] * slots * _width(c)
    if c["kind"] == "choose":
        code = d if c["fmt"] == "e4m3" else 2 * d
        touched = sum(length - (length - n) // c["page"] * c["page"] for n, length in _sizes(c))
        pages = sum(-(-length // c["page"]) for _, length in _sizes(c))
        return {"bytes": 2 * d * rows * c["Hq"] + c["Hkv"] * (touched * code + pages * (d + 1)) + lists,
                "flops": sum(2 * d * m * whole for _, _, m, _, _, whole, _ in tiles) * c["Hq"]}
    keys, pairs = [0] * c["B"], 0
    for b, _, m, _, lo, whole, own_last in tiles:
        see = min(_width(c), max(whole, own_last + 1)) * c["page"]
        keys[b] += see
        pairs += m * see
    held = sum(min(k, length) for k, (_, length) in zip(keys, _sizes(c)))
    return {"bytes": held * c["Hkv"] * row + 4 * d * rows * c["Hq"] + lists, "flops": 4 * d * pairs * c["Hq"]}


def _cost(c):
    """About the seconds of a pass."""
    w = work(c)
    return w["flops"] / 1e15 + w["bytes"] / 5e12


# ---------------------------------------------------------------- the cache in plain torch
def _quantise(x):
    """e4m3 codes and scale bytes of rows x [.., d]."""
    x = x.float()
    m, q = torch.frexp(x.abs().amax(-1))
    e = torch.where(m <= 0.875, q - 9, q - 8)                 # the smallest e with max |x| <= 448 * 2^e = 0.875 * 2^(e + 9)
    e = torch.where(m > 0, e.clamp(min=EMIN), torch.zeros_like(e))
    return torch.ldexp(x, -e[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _raw(pool):
    return pool.view(torch.uint8) if pool.dtype == torch.float8_e4m3fn else pool


def _rows_of(pool, scales, page, slot, dtype=torch.float32):
    """Rows [n][H][d] of the pool in 32 bits (or more)."""
    x = _raw(pool)[page, :, slot].view(pool.dtype).to(dtype)
    if scales is None:
        return x
    return x * torch.ldexp(torch.ones_like(x[..., 0]), scales[page, :, slot].int() - 127)[..., None]


def _pools(s):
    out = [(s["k"], s["ks"]), (s["v"], s["vs"])]
    return out


def _pool(s):
    return {"k": s["k"], "v": s["v"]} if s["ks"] is None else {"k": s["k"], "v": s["v"], "ks": s["ks"], "vs": s["vs"]}


def _copy_rows(s, src_page, src_slot, dst_page, dst_slot):
    for pool, scales in _pools(s):
        _raw(pool)[dst_page, :, dst_slot] = _raw(pool)[src_page, :, src_slot]
        if scales is not None:
            scales[dst_page, :, dst_slot] = scales[src_page, :, src_slot]


# ---------------------------------------------------------------- norm and rotation
def _rotate(s, x, weight, dtype):
    """x [H][rows][d] normed by head and rotated to its coordinates, in `dtype`; the angles in 64 bits."""
    c, d = s["case"], s["case"]["d"]
    x = x.to(dtype)
    if c["norm"]:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * weight.to(dtype)
    a = s["coord"].double()[s["axis"]].T * s["theta"].double()          # [rows][d / 2]
    cos, sin = torch.cos(a).to(dtype), torch.sin(a).to(dtype)
    if c["half"]:
        p, q = x[..., :d // 2], x[..., d // 2:]
        return torch.cat([p * cos - q * sin, p * sin + q * cos], -1)
    p, q = x[..., 0::2], x[..., 1::2]
    return torch.stack([p * cos - q * sin, p * sin + q * cos], -1).flatten(-2)


def _plain_rope(s):
    q = _rotate(s, s["q"], s["qw"], torch.float32).to(torch.bfloat16)
    k = _rotate(s, s["kn"], s["kw"], torch.float32).to(torch.bfloat16)
    if s["case"]["dense"]:
        return {"q": q, "k_rows": k}
    page, slot = s["table"][s["seq"], s["pos"] // s["case"]["page"]].long(), s["pos"] % s["case"]["page"]
    for pool, scales, x in ((s["k"], s["ks"], k), (s["v"], s["vs"], s["vn"])):
        x = x.transpose(0, 1)
        if scales is None:
            pool[page, :, slot] = x
        else:
            codes, byte = _quantise(x)
            _raw(pool)[page, :, slot] = codes.view(torch.uint8)
            scales[page, :, slot] = byte
    return {"q": q, **_pool(s)}


# ---------------------------------------------------------------- pages
def _plain_fork(s):
    c, page, n_pages = s["case"], s["case"]["page"], s["k"].shape[0]
    refs = s["refs"]
    refs.copy_(s["refs0"])
    on, parent = s["parent"] >= 0, s["parent"].clamp(min=0).long()
    table = torch.where(on[:, None], s["table"][parent], -1)
    length = torch.where(on, s["seq_len"][parent], 0)
    children = torch.zeros_like(s["seq_len"]).scatter_add_(0, parent, on.to(torch.int32))
    held = s["table"] >= 0
    refs.index_add_(0, s["table"][held].long(), (children[:, None] - 1).expand(held.shape)[held])
    # room for the new tokens
    new, k = length + s["add"], torch.arange(table.shape[1], device="cuda")
    grow, first = s["add"] > 0, (length // page).long()
    last = table.gather(1, first.clamp(max=table.shape[1] - 1)[:, None])[:, 0]
    part = grow & (length % page > 0)
    at = torch.where(part, last, n_pages).long()
    here = torch.zeros(n_pages + 1, dtype=torch.int64, device="cuda").index_add_(0, at, torch.ones_like(at))
    b = torch.arange(c["B2"], device="cuda")
    highest = torch.full((n_pages + 1,), -1, dtype=torch.int64, device="cuda").scatter_reduce_(0, at, b, "amax")
    count = torch.cat([refs, refs.new_zeros(1)])[at]
    copied = part & (count > 1) & ~((highest[at] == b) & (here[at] == count))
    need = grow[:, None] & (k >= -(-length // page)[:, None]) & (k < -(-new // page)[:, None])
    need |= copied[:, None] & (k == first[:, None])
    rank = (need.flatten().cumsum(0) - 1).view(need.shape)
    free = torch.argsort((refs > 0).to(torch.int32), stable=True).to(torch.int32)
    table = torch.where(need, free[rank.clamp(min=0)], table)
    refs.index_add_(0, at[copied], torch.full_like(at[copied], -1, dtype=torch.int32))
    refs.index_add_(0, table[need].long(), torch.ones_like(table[need]))
    src, dst = last[copied].long(), table[copied, first[copied]].long()
    slot = torch.arange(page, device="cuda")
    i, j = torch.nonzero(slot < (length % page)[copied][:, None], as_tuple=True)
    _copy_rows(s, src[i], j, dst[i], j)
    return {"table": table, "seq_len": new, "refs": refs, **_pool(s)}


def _plain_compact(s):
    page = s["case"]["page"]
    refs, old = s["refs"], s["table"]
    refs.copy_(s["refs0"])
    keep, seq, pos = s["keep"].long(), s["kept_seq"], s["kept_pos"]
    n = (s["keep_start"][1:] - s["keep_start"][:-1]).to(torch.int32)
    moved = torch.where(keep == pos, torch.full_like(pos, 1 << 40), pos)
    same = n.long().scatter_reduce(0, seq, moved, "amin")     # leading positions that stay where they are
    k = torch.arange(old.shape[1], device="cuda")
    end = torch.minimum((k + 1) * page, n.long()[:, None])
    used = k * page < n[:, None]
    stay, fresh = used & (end <= same[:, None]), used & (end > same[:, None])
    rank = (fresh.flatten().cumsum(0) - 1).view(fresh.shape)
    free = torch.argsort((refs > 0).to(torch.int32), stable=True).to(torch.int32)
    table = torch.where(stay, old, torch.where(fresh, free[rank.clamp(min=0)], torch.full_like(old, -1)))
    gone = (old >= 0) & ~stay
    refs.index_add_(0, old[gone].long(), torch.full_like(old[gone], -1))
    refs.index_add_(0, table[fresh].long(), torch.ones_like(table[fresh]))
    go = fresh[seq, pos // page]
    seq, pos, keep = seq[go], pos[go], keep[go]
    _copy_rows(s, old[seq, keep // page].long(), keep % page, table[seq, pos // page].long(), pos % page)
    return {"table": table, "seq_len": n, "refs": refs, **_pool(s)}


# ---------------------------------------------------------------- summaries and choice
def _codes8(x):
    """Integers c and exponents e of rows x [.., d] in 64 bits: c = x 2^-e to nearest, e the smallest >= SMIN with
    max |x| <= 127 2^e; rows that are not finite or reach WILD have no use."""
    a = x.abs().amax(-1)
    wild = ~(a < WILD)
    m, q = torch.frexp(torch.where(wild, torch.zeros_like(a), a))
    e = torch.where(m <= 0.9921875, q - 7, q - 6)
    e = torch.where(m > 0, e.clamp(min=SMIN), torch.full_like(e, SMIN))
    x = torch.where(wild[..., None], torch.zeros_like(x), x)
    return torch.round(torch.ldexp(x, -e[..., None])), e, wild


def _plain_summarise(s, seq, k):
    """Summaries of page k[i] of sequence seq[i]."""
    page = s["case"]["page"]
    at = s["table"][seq, k].long()
    held = (s["seq_len"][seq].long() - k * page).clamp(max=page)
    for i in range(0, at.numel(), 256):
        z = slice(i, i + 256)
        x = _raw(s["k"])[at[z]].view(s["k"].dtype).double()                  # [n][H][page][d]
        if s["ks"] is not None:
            x = x * torch.ldexp(torch.ones_like(x[..., 0]), s["ks"][at[z]].int() - 127)[..., None]
        on = torch.arange(page, device="cuda") < held[z, None]
        x = torch.where(on[:, None, :, None], x, torch.zeros_like(x))
        c, e, wild = _codes8(x.sum(2) / held[z, None, None])
        s["code"][at[z]] = c.to(torch.int8)
        s["scale"][at[z]] = torch.where(wild, torch.full_like(e, 255), e + 127).to(torch.uint8)


def _plain_choose(s):
    c = s["case"]
    page, H, G, d = c["page"], c["Hkv"], c["Hq"] // c["Hkv"], c["d"]
    _plain_summarise(s, s["touch_seq"], s["touch_page"])
    lists = torch.full((H, s["slots"], s["width"]), -1, dtype=torch.int32, device="cuda")
    cq, eq, wild = _codes8(s["q"].double())
    cq, eq = cq.float(), eq.int()
    for b, (n, length) in enumerate(s["sizes"]):
        np = -(-length // page)
        at = s["table"][b, :np].long()
        lo, hi = s["bounds"][b]
        code, byte = s["code"][at].float(), s["scale"][at]                   # [np][H][d]
        unit = torch.where(byte == 255, torch.zeros_like(byte, dtype=torch.float32),
                           torch.ldexp(torch.ones_like(byte, dtype=torch.float32), byte.int() - 127))
        k = torch.arange(np, device="cuda")
        t_first, t_slot, t_lo, t_whole, t_own = s["tiles"][b]
        tiles = t_first.numel()
        for h in range(H):
            best = torch.full((tiles * c["tile"], np), -math.inf, device="cuda")
            for g in range(G):
                r = h * G + g
                x = cq[r, lo:hi] @ code[:, h].T                              # whole numbers below 2^24: exact
                x = torch.ldexp(x, eq[r, lo:hi, None]).masked_fill_(wild[r, lo:hi, None], -math.inf)
                best[:n] = torch.maximum(best[:n], x)
            score = best.view(tiles, c["tile"], np).amax(1)
            score = torch.where(score == -math.inf, score, score * unit[:, h])
            score = score.masked_fill_((byte[:, h] == 255)[None], -math.inf)
            local = (k >= t_lo[:, None]) & (k <= t_own[:, None])
            seen = k < t_whole[:, None]
            forced = local | (seen & (k < c["sink_pages"]))
            score = score.masked_fill_(~seen | forced, -math.inf)
            top, order = torch.sort(score, dim=1, descending=True, stable=True)
            m = min(c["top"], np)
            pick = torch.zeros(tiles, np, dtype=torch.bool, device="cuda")
            pick.scatter_(1, order[:, :m], top[:, :m] > -math.inf)
            pick |= forced
            line = torch.where(pick, k, np).sort(1)[0][:, :s["width"]]
            lists[h, t_slot, :line.shape[1]] = torch.where(line < np, line, -1).to(torch.int32)
    return {"code": s["code"], "scale": s["scale"], "lists": lists}


# ---------------------------------------------------------------- attention over chosen pages
def _plain_chosen(s):
    c = s["case"]
    page, H, G, d, tile = c["page"], c["Hkv"], c["Hq"] // c["Hkv"], c["d"], c["tile"]
    out = torch.empty_like(s["q"])
    slot = torch.arange(page, device="cuda")
    for b, (n, length) in enumerate(s["sizes"]):
        lo, hi = s["bounds"][b]
        if n == 0:
            continue
        _, t_slot, _, _, _ = s["tiles"][b]
        tiles = t_slot.numel()
        p = length - n + torch.arange(tiles * tile, device="cuda").view(tiles, tile)
        end = torch.full_like(p, length) if c["block"] == 0 else ((p // c["block"] + 1) * c["block"]).clamp(max=length)
        q = torch.zeros(c["Hq"], tiles * tile, d, device="cuda")
        q[:, :n] = s["q"][:, lo:hi].float()
        q = q.view(H, G, tiles, tile, d)
        step = max(1, int(4e8 // (H * s["width"] * page * d)))
        for t in range(0, tiles, step):
            z = slice(t, min(t + step, tiles))
            entry = s["lists"][:, t_slot[z]].long()                          # [H][tiles][width]
            pos = entry[..., None] * page + slot                             # [H][tiles][width][page]
            see = (entry >= 0)[..., None] & (pos < length)
            at = s["table"][b, entry.clamp(min=0)].long()
            h = torch.arange(H, device="cuda")[:, None, None]
            kv = []
            for pool, scales in _pools(s):
                x = _raw(pool)[at, h].view(pool.dtype).float()               # [H][tiles][width][page][d]
                if scales is not None:
                    x = x * torch.ldexp(torch.ones_like(x[..., 0]), scales[at, h].int() - 127)[..., None]
                kv.append(x.flatten(2, 3))
            pos, see = pos.flatten(2), see.flatten(2)
            qz = q[:, :, z].permute(0, 2, 1, 3, 4)                           # [H][tiles][G][tile][d]
            score = (qz.flatten(2, 3) @ kv[0].transpose(-1, -2)).mul_(1.0 / math.sqrt(d)).view(*qz.shape[:4], -1)
            ok = see[:, :, None] & (pos[:, :, None] < end[z][None, :, :, None])
            score = score.masked_fill_(~ok[:, :, None], -math.inf)
            top = score.amax(-1, keepdim=True)
            score = score.sub_(torch.where(torch.isfinite(top), top, torch.zeros_like(top))).exp_()
            total = score.sum(-1, keepdim=True)
            o = (score.flatten(2, 3) @ kv[1]).view(qz.shape) / torch.where(total > 0, total, torch.ones_like(total))
            o = o.permute(0, 2, 1, 3, 4).reshape(c["Hq"], -1, d)             # rows of the tiles z
            m = min(n - t * tile, o.shape[1])
            out[:, lo + t * tile:lo + t * tile + m] = o[:, :m].to(out.dtype)
    return {"o": out}


# ---------------------------------------------------------------- inputs
def _keys(c, gen, *shape):
    """Rows of norm about sqrt(d) around 64 centres for each head (the heads are dimension 1), as post-rotary keys
    and queries are."""
    d, heads = c["d"], shape[1]
    mu = torch.randn(heads, 64, d, generator=gen, device="cuda")
    which = torch.randint(0, 64, shape, generator=gen, device="cuda")
    head = torch.arange(heads, device="cuda").view(1, heads, *([1] * (len(shape) - 2))).expand(shape)
    x = mu[head, which].mul_(0.9)
    return x.add_(torch.randn(x.shape, generator=gen, device="cuda"), alpha=0.44).to(torch.bfloat16)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def prepare(c, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    sizes = _sizes(c)
    T, H, d, page = sum(n for n, _ in sizes), c["Hkv"], c["d"], c["page"]
    starts = [0]
    for n, _ in sizes:
        starts.append(starts[-1] + n)
    s = {"case": c, "sizes": sizes, "ks": None, "vs": None, "seq_len": _i32([length for _, length in sizes]),
         "row_start": _i32(starts), "bounds": [(starts[b], starts[b + 1]) for b in range(c["B"])]}
    s["seq"] = torch.repeat_interleave(torch.arange(c["B"], device="cuda"), _i32([n for n, _ in sizes]))
    first = _i32([length - n for n, length in sizes])
    s["pos"] = (first[s["seq"]] + torch.arange(T, device="cuda") - s["row_start"][s["seq"]]).to(torch.int32)
    if c["kind"] == "rope":
        _prepare_rope(c, gen, s, T)
        if c["dense"]:
            return s
    # ---- pages: of every sequence, of what it is to grow by, and some in nobody's hands
    held = [length for _, length in sizes]
    pages, cols, more = [-(-x // page) for x in held], 1, 3
    if c["kind"] == "fork":
        parents, add = _parents(c)
        ends = [(held[p] if p >= 0 else 0, (held[p] if p >= 0 else 0) + x) for p, x in zip(parents, add)]
        cols = max(-(-z // page) for _, z in ends)
        more += sum(-(-z // page) - a // page for a, z in ends)
    kept = _kept(c) if c["kind"] == "compact" else []
    more += sum(-(-len(x) // page) for x in kept)
    cols = max([1, cols] + pages + [-(-len(x) // page) for x in kept])
    total = sum(pages) + more
    order = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((c["B"], cols), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, m in enumerate(pages):
        table[b, :m] = order[at:at + m]
        at += m
    s["table"] = table
    if c["kind"] == "rope":
        s["k"] = torch.zeros(total, H, page, d, dtype=torch.bfloat16, device="cuda")
        s["v"] = s["k"].clone()
    else:
        s["k"] = _keys(c, gen, total, H, page)
        s["v"] = torch.randn(total, H, page, d, generator=gen, device="cuda", dtype=torch.bfloat16)
    if c["fmt"] == "e4m3":
        (s["k"], s["ks"]), (s["v"], s["vs"]) = _quantise(s["k"]), _quantise(s["v"])
    if c["kind"] in ("fork", "compact"):
        s["refs0"] = torch.zeros(total, dtype=torch.int32, device="cuda")
        s["refs0"][table[table >= 0].long()] = 1
        s["refs"] = s["refs0"].clone()
    if c["kind"] == "fork":
        s["parent"], s["add"] = _i32(parents), _i32(add)
    if c["kind"] == "compact":
        s["keep"] = _i32([j for x in kept for j in x])
        at = [0]
        for x in kept:
            at.append(at[-1] + len(x))
        s["keep_start"] = _i32(at)
        s["kept_seq"] = torch.repeat_interleave(torch.arange(c["B"], device="cuda"), _i32([len(x) for x in kept]))
        s["kept_pos"] = torch.arange(at[-1], device="cuda") - s["keep_start"][s["kept_seq"]].long()
    if c["kind"] in ("choose", "chosen"):
        s["q"] = _keys(c, gen, T, c["Hq"]).transpose(0, 1).contiguous()
        tiles, s["slots"] = _tiles(c)
        s["width"] = _width(c)
        s["tiles"] = []
        for b in range(c["B"]):
            mine = [t for t in tiles if t[0] == b]
            s["tiles"].append([torch.tensor([t[i] for t in mine], dtype=torch.int64, device="cuda") for i in (1, 3, 4, 5, 6)])
    if c["kind"] == "choose":
        s["code"] = torch.zeros(total, H, d, dtype=torch.int8, device="cuda")
        s["scale"] = torch.full((total, H), 127, dtype=torch.uint8, device="cuda")
        every = [(b, k) for b, m in enumerate(pages) for k in range(m)]
        _plain_summarise(s, *(torch.tensor(x, device="cuda") for x in zip(*every)))
        new = [(b, k) for b, (n, length) in enumerate(sizes) for k in range((length - n) // page, pages[b])]
        s["touch_seq"], s["touch_page"] = (torch.tensor(x, device="cuda") for x in zip(*new))
    if c["kind"] == "chosen":
        s["lists"] = _random_lists(c, gen, s, pages)
    if own:
        from paper_2608_27922_gb300 import dkv
        s["cache"] = dkv.PagedCache(H, d, page, total, c["fmt"], k=s["k"], v=s["v"], k_scale=s["ks"], v_scale=s["vs"])
        s["seqs"] = dkv.CacheSeqs(table, s["seq_len"], s["row_start"])
        if c["kind"] in ("fork", "compact"):
            s["pages"] = dkv.PageTable(table, s["seq_len"])
            n = c["B2"] if c["kind"] == "fork" else c["B"]
            s["to"] = dkv.PageTable(torch.full((n, cols), -1, dtype=torch.int32, device="cuda"), _i32([0] * n))
        if c["kind"] == "choose":
            s["summaries"] = dkv.Summaries(s["cache"], code=s["code"], scale=s["scale"])
    return s


def _prepare_rope(c, gen, s, T):
    H, d = c["Hkv"], c["d"]
    # rows of different magnitudes, as projections give them
    size = lambda heads: torch.exp2(torch.randint(-3, 4, (heads, T, 1), generator=gen, device="cuda").float())
    s["q"] = (_keys(c, gen, T, c["Hq"]).transpose(0, 1) * size(c["Hq"])).to(torch.bfloat16).contiguous()
    s["kn"] = (_keys(c, gen, T, H).transpose(0, 1) * size(H)).to(torch.bfloat16).contiguous()
    s["vn"] = torch.randn(H, T, d, generator=gen, device="cuda", dtype=torch.bfloat16)
    s["qw"] = 1.0 + 0.2 * torch.randn(d, generator=gen, device="cuda")
    s["kw"] = 1.0 + 0.2 * torch.randn(d, generator=gen, device="cuda")
    s["eps"] = 1e-6
    # the pairs of each axis (time, row, column: the first has what is left over) and their frequencies
    rest = d // 2 // c["axes"]
    s["pairs"] = [d // 2 - rest * (c["axes"] - 1)] + [rest] * (c["axes"] - 1)
    s["axis"] = torch.tensor([a for a, m in enumerate(s["pairs"]) for _ in range(m)], device="cuda")
    s["theta"] = torch.tensor([10000.0 ** (-j / m) for m in s["pairs"] for j in range(m)], device="cuda")
    if c["axes"] == 1:
        s["coord"] = s["pos"][None].clone()
    else:                                                     # frames of 30 x 52
        s["coord"] = torch.stack([s["pos"] // 1560, s["pos"] % 1560 // 52, s["pos"] % 52]).to(torch.int32)
    if own:
        from paper_2608_27922_gb300 import dkv
        s["how"] = dkv.NormRope(d, s["theta"], axis_pairs=s["pairs"],
                                layout=dkv.DKV_ROPE_HALF if c["half"] else dkv.DKV_ROPE_INTERLEAVED, norm=c["norm"],
                                eps=s["eps"], q_weight=s["qw"], k_weight=s["kw"])


def _random_lists(c, gen, s, pages):
    lists = torch.full((c["Hkv"], s["slots"], s["width"]), -1, dtype=torch.int32, device="cuda")
    for b, m in enumerate(pages):
        _, t_slot, t_lo, t_whole, t_own = s["tiles"][b]
        if not t_slot.numel():
            continue
        k = torch.arange(m, device="cuda")
        x = torch.rand(c["Hkv"], t_slot.numel(), m, generator=gen, device="cuda")
        local = (k >= t_lo[:, None]) & (k <= t_own[:, None])
        seen = k < t_whole[:, None]
        forced = local | (seen & (k < c["sink_pages"]))
        x = torch.where(forced, 2.0 + x, torch.where(seen, x, torch.full_like(x, -1.0)))
        room = c["top"] + forced.sum(-1)                      # [tiles]
        x, order = x.sort(-1, descending=True)
        line = torch.where((x >= 0) & (k < room[:, None]), order, m).sort(-1)[0][..., :s["width"]]
        lists[:, t_slot, :line.shape[-1]] = torch.where(line < m, line, -1).to(torch.int32)
    return lists


def run(s):
    c = s["case"]
    if c["kind"] == "rope":
        if not own:
            return _plain_rope(s)
        if c["dense"]:
            from paper_2608_27922_gb300 import dkv
            q, k = dkv.norm_rope(s["q"], s["kn"], s["how"], s["coord"])
            return {"q": q, "k_rows": k}
        q = s["cache"].write_norm_rope(s["q"], s["kn"], s["vn"], s["seqs"], s["how"], coord=None if c["axes"] == 1 else s["coord"])
        return {"q": q, **_pool(s)}
    if c["kind"] == "fork":
        if not own:
            return _plain_fork(s)
        s["refs"].copy_(s["refs0"])                           # (so that a pass can be repeated)
        s["cache"].fork(s["refs"], s["pages"], s["parent"], s["to"])
        s["cache"].extend(s["refs"], s["to"], s["add"])
        return {"table": s["to"].block_table, "seq_len": s["to"].seq_len, "refs": s["refs"], **_pool(s)}
    if c["kind"] == "compact":
        if not own:
            return _plain_compact(s)
        s["refs"].copy_(s["refs0"])
        s["cache"].compact(s["refs"], s["pages"], s["keep"], s["keep_start"], s["to"])
        return {"table": s["to"].block_table, "seq_len": s["to"].seq_len, "refs": s["refs"], **_pool(s)}
    if c["kind"] == "choose":
        if not own:
            return _plain_choose(s)
        s["cache"].summarise(s["seqs"], s["summaries"])
        lists = s["cache"].choose(s["q"], s["seqs"], s["summaries"], c["top"], tile=c["tile"], block=c["block"],
                                  sink_pages=c["sink_pages"], local_pages=c["local_pages"])
        return {"code": s["code"], "scale": s["scale"], "lists": lists}
    if own:
        return {"o": s["cache"].attend_chosen(s["q"], s["seqs"], s["lists"], tile=c["tile"], block=c["block"])}
    return _plain_chosen(s)


# ---------------------------------------------------------------- the definition in 64 bits
def _decode(codes, scale):
    """Values of e4m3 codes (sign, 4 exponent bits of bias 7, 3 mantissa bits) times their row's scale."""
    b = codes.view(torch.uint8).to(torch.int64)
    e, m = (b >> 3) & 15, (b & 7).double()
    x = torch.where(e > 0, (8 + m) * torch.exp2((e - 10).double()), m * 2.0 ** -9) * torch.where(b > 127, -1.0, 1.0)
    return x * torch.exp2((scale.to(torch.int64) - 127).double())[..., None]


def exact(c, seed):
    s = prepare(c, seed)
    return {"rope": _exact_rope, "fork": _exact_fork, "compact": _exact_compact, "choose": _exact_choose,
            "chosen": _exact_chosen}[c["kind"]](s)


class _Book:
    """Tables, lengths and counts as lists, and the page copies that come of what is done to them, one after the other."""

    def __init__(self, s):
        self.s, self.page = s, s["case"]["page"]
        self.table, self.length, self.refs = (s[x].tolist() for x in ("table", "seq_len", "refs0"))
        self.free = [p for p, r in enumerate(self.refs) if r == 0]
        self.moves = []                                       # (page, first slot, page, first slot, rows)

    def take(self):
        p = self.free.pop(0)
        self.refs[p] += 1
        return p

    def done(self, table, length):
        cols = self.s["table"].shape[1]
        table = _i32([row + [-1] * (cols - len(row)) for row in table])
        pools = _pool(self.s)
        out = {name: pool.clone() for name, pool in pools.items()}
        for a, i, z, j, n in self.moves:
            for name, pool in pools.items():
                _raw(out[name])[z, :, j:j + n] = _raw(pool)[a, :, i:i + n]
        out = {name: x if x.dtype == torch.uint8 else x.double() for name, x in out.items()}
        return {"table": table, "seq_len": _i32(length), "refs": _i32(self.refs), **out}


def _exact_fork(s):
    book, page = _Book(s), s["case"]["page"]
    parents, add = s["parent"].tolist(), s["add"].tolist()
    table = [[p for p in book.table[a] if p >= 0] if a >= 0 else [] for a in parents]
    length = [book.length[a] if a >= 0 else 0 for a in parents]
    for row in book.table:
        for p in row:
            if p >= 0:
                book.refs[p] -= 1
    for row in table:
        for p in row:
            book.refs[p] += 1
    book.free = [p for p, r in enumerate(book.refs) if r == 0]
    for b, row in enumerate(table):
        new = length[b] + add[b]
        if add[b] and length[b] % page and book.refs[row[-1]] > 1:
            src = row[-1]                                     # others hold it still: this one goes on in a copy
            book.refs[src] -= 1
            row[-1] = book.take()
            book.moves.append((src, 0, row[-1], 0, length[b] % page))
        while len(row) * page < new:
            row.append(book.take())
        length[b] = new
    return book.done(table, length)


def _exact_compact(s):
    book, page = _Book(s), s["case"]["page"]
    keep, start, table, gone = s["keep"].tolist(), s["keep_start"].tolist(), [], []
    for b, old in enumerate(book.table):
        mine, row = keep[start[b]:start[b + 1]], []
        for k in range(0, len(mine), page):
            part = mine[k:k + page]
            if row == old[:len(row)] and part == list(range(k, k + len(part))):
                row.append(old[k // page])
                continue
            row.append(book.take())
            book.moves += [(old[j // page], j % page, row[-1], i, 1) for i, j in enumerate(part)]
        gone += [p for k, p in enumerate(old) if p >= 0 and not (k < len(row) and row[k] == p)]
        table.append(row)
    for p in gone:
        book.refs[p] -= 1
    return book.done(table, [z - a for a, z in zip(start, start[1:])]) if len(book.moves) < 60000 else None


def _exact_choose(s):
    """In whole numbers: scores as integers times powers of two, compared in 64 bits."""
    c = s["case"]
    if work(c)["flops"] > 3e9:
        return None
    G, page = c["Hq"] // c["Hkv"], c["page"]
    code, scale = s["code"].clone(), s["scale"].clone()

    def eight(x):
        a = x.abs().amax(-1)
        fine = a < WILD                                       # (not so for a NaN)
        e = torch.full(a.shape, SMIN, dtype=torch.int64, device="cuda")
        for step in (64, 32, 16, 8, 4, 2, 1):                 # the smallest e that holds, by halves
            e = torch.where(a > 127 * torch.exp2((e + step - 1).double()), e + step, e)
        return torch.where(fine[..., None], (x * torch.exp2(-e.double())[..., None]).round(), 0.0), e, fine

    for b, (n, length) in enumerate(s["sizes"]):
        for k in range((length - n) // page, -(-length // page)):
            p, m = int(s["table"][b, k]), min(page, length - k * page)
            x = s["k"][p, :, :m].double() if s["ks"] is None else _decode(s["k"].view(torch.uint8)[p, :, :m], s["ks"][p, :, :m])
            v, e, fine = eight(x.sum(1) / m)
            code[p], scale[p] = v.to(torch.int8), torch.where(fine, e + 127, 255).to(torch.uint8)
    lists = torch.full((c["Hkv"], s["slots"], s["width"]), -1, dtype=torch.int32)
    qc, qe, q_fine = eight(s["q"].double())
    for b, i, m, slot, lo, whole, own_last in _tiles(c)[0]:
        at = s["bounds"][b][0] + i
        p = s["table"][b, :whole].long()
        x = torch.einsum("hgmd,phd->hgmp", qc[:, at:at + m].view(c["Hkv"], G, m, -1), code[p].double())
        x = x * torch.exp2(qe[:, at:at + m].view(c["Hkv"], G, m, 1).double())
        x = torch.where(q_fine[:, at:at + m].view(c["Hkv"], G, m, 1), x, -math.inf).amax((1, 2))
        byte = scale[p].T
        x = torch.where((byte != 255) & (x > -math.inf), x * torch.exp2(byte.double() - 127), -math.inf).tolist()
        for h, line in enumerate(x):
            forced = {k for k in range(whole) if k < c["sink_pages"]} | set(range(lo, own_last + 1))
            rest = sorted((-v, k) for k, v in enumerate(line) if v > -math.inf and k not in forced)[:c["top"]]
            row = sorted(forced | {k for _, k in rest})
            lists[h, slot, :len(row)] = torch.tensor(row, dtype=torch.int32)
    return {"code": code, "scale": scale, "lists": lists.cuda()}


def _exact_rope(s):
    """Rows by complex numbers; of a quantised row the values that its codes stand for before they are rounded."""
    c, d = s["case"], s["case"]["d"]
    turn = torch.polar(torch.ones(s["coord"].shape[1], d // 2, dtype=torch.float64, device="cuda"),
                       torch.stack([s["coord"][a].double() * s["theta"][j].double() for j, a in enumerate(s["axis"].tolist())], 1))
    rows = {}
    for name, x, w in (("q", s["q"], s["qw"]), ("k_rows", s["kn"], s["kw"])):
        x = x.double()
        if c["norm"]:
            x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / d + s["eps"]) * w.double()
        pair = x.unflatten(-1, (2, d // 2)).transpose(-1, -2) if c["half"] else x.unflatten(-1, (d // 2, 2))
        z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
        rows[name] = (z.transpose(-1, -2) if c["half"] else z).flatten(-2)
    if c["dense"]:
        return rows
    out = {"q": rows["q"]}
    at = s["pos"].long()
    page = s["table"][s["seq"], at // c["page"]].long()
    for name, x in (("k", rows["k_rows"]), ("v", s["vn"].double())):
        x, pool = x.transpose(0, 1), s[name].double()
        if s["ks"] is not None:
            x = x.to(torch.bfloat16).double()
            top = x.abs().amax(-1, keepdim=True)
            e = torch.where(top > 0, torch.ceil(torch.log2(top / 448.0)).clamp(min=EMIN), torch.zeros_like(top))
            x = x * torch.exp2(-e)
            out[name + "s"] = None
        pool[page, :, at % c["page"]] = x
        out[name] = pool
    return out


def _exact_chosen(s):
    c = s["case"]
    if work(c)["flops"] > 2e12 or s["lists"].shape[0] * s["lists"].shape[1] > 6000:
        return None
    G, page = c["Hq"] // c["Hkv"], c["page"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lists = s["lists"].tolist()
    for b, i, m, slot, _, _, _ in _tiles(c)[0]:
        n, length = s["sizes"][b]
        p = torch.arange(length - n + i, length - n + i + m, device="cuda")
        end = torch.full_like(p, length) if c["block"] == 0 else ((p // c["block"] + 1) * c["block"]).clamp(max=length)
        z = slice(s["bounds"][b][0] + i, s["bounds"][b][0] + i + m)
        for h in range(c["Hkv"]):
            entries = torch.tensor([x for x in lists[h][slot] if x >= 0], device="cuda")
            j = (entries[:, None] * page + torch.arange(page, device="cuda")).flatten()
            j = j[j < length]
            at, off = s["table"][b, j // page].long(), j % page
            kv = []
            for pool, scales in _pools(s):
                x = pool.view(torch.uint8)[at, h, off] if scales is not None else pool[at, h, off].double()
                kv.append(x if scales is None else _decode(x, scales[at, h, off]))
            x = s["q"][h * G:(h + 1) * G, z].double() @ kv[0].T / math.sqrt(c["d"])
            x = x.masked_fill(j[None] >= end[:, None], -math.inf)
            out[h * G:(h + 1) * G, z] = torch.softmax(x, -1) @ kv[1]
    return {"o": out}
