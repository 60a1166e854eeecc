"""The paged cache of a window's keys and values, as cases to time and compare.

  write    dkv_cache_write: the newest tokens' keys and values into their pages, as they are (bf16) or
           quantised (e4m3 codes, one power-of-two scale for each row of d values);
  read     dkv_cache_read: a range of each sequence back as dense bf16 rows, which is how a block that
           leaves the window reaches the bank;
  attend   dkv_cache_attend: the newest tokens' queries over their sequence's cached keys, causal by
           blocks of tokens, with a sliding window and sinks, grouped heads and a ragged batch.

Sequence b holds L tokens; its n newest are rows [row_start[b], row_start[b + 1]) of the packed
tensors [heads][rows][d], at positions L - n .. L - 1.  Position j is slot j % page_len of page
table[b][j / page_len]; a page is [heads][page_len][d].  With end(p) = the end of p's block of `block`
tokens (block 0: of the sequence), position j is visible from p when j < end(p) and j is one of the
last `window` positions before end(p) (window 0: no limit) or one of the first `sinks`.
"""
import math
import random

import torch

own = False

EMIN = -110                      # smallest exponent of a scale: codes times scale stay normal bf16 numbers

_BASE = dict(kind="attend", fmt="bf16", d=128, page=64, Hq=12, Hkv=12, B=1, n_lo=1, n_hi=1, past_lo=0, past_hi=0,
             window=0, sinks=0, block=1, mix=0)


def _case(**kw):
    c = dict(_BASE)
    c.update(kw)
    return c


def listed():
    return [
        # One new token of one sequence, a frame of 1,560 tokens behind it: the smallest call, launches count.
        _case(name="token_small", past_lo=1560, past_hi=1560),
        # One new token each of 32 sequences, grouped heads (five query heads a key head), quantised cache of ragged
        # lengths: a server's steady state.
        _case(name="token_batch", fmt="e4m3", Hq=40, Hkv=8, B=32, past_lo=700, past_hi=9360, mix=1),
        # One new token over a very long cache: the keys have to be split over the whole GPU.
        _case(name="token_long", page=128, past_lo=131000, past_hi=131000),
        # Five tokens at a time (drafted ones to be checked), small pages, a window that leaves most of a long cache out.
        _case(name="draft_window", page=16, Hq=12, Hkv=4, B=8, n_lo=2, n_hi=5, past_lo=90, past_hi=20000, window=2048,
              sinks=4, mix=2),
        # A 3-frame block's queries over the sink frame, the window and their own block, quantised; most of the
        # 30-frame cache is hidden.
        _case(name="block_window", fmt="e4m3", n_lo=4680, n_hi=4680, past_lo=42120, past_hi=42120, window=12480,
              sinks=1560, block=4680),
        # A layer of 40 heads: a block's queries over a 9,360-token past and themselves, no mask inside the block.
        _case(name="stack_block", page=128, Hq=40, Hkv=40, n_lo=4680, n_hi=4680, past_lo=9360, past_hi=9360, block=0),
        # Prompts of three sequences at once, causal, ragged, grouped heads, each behind a cached part.
        _case(name="prompt_causal", page=32, Hq=40, Hkv=8, B=3, n_lo=900, n_hi=2600, past_lo=0, past_hi=2900, mix=3),
        # Chunks of a small model's text (64 dimensions, three query heads a key head), quantised, short window.
        _case(name="chunk_window_d64", fmt="e4m3", d=64, page=16, Hq=24, Hkv=8, B=4, n_lo=333, n_hi=700, past_lo=0,
              past_hi=7600, window=1024, sinks=16, mix=4),
        # A frame of one layer written as it is.
        _case(name="frame_write", kind="write", page=128, n_lo=1560, n_hi=1560, past_lo=7800, past_hi=7800),
        # A block of four stacked layers of 40 heads, quantised on its way in.
        _case(name="stack_write", kind="write", fmt="e4m3", Hq=160, Hkv=160, n_lo=4680, n_hi=4680, past_lo=4703,
              past_hi=4703),
        # A frame of one layer read back, pages of 16.
        _case(name="frame_read", kind="read", page=16, n_lo=1560, n_hi=1560, past_lo=7801, past_hi=7801),
        # The block of those stacked layers that leaves the window, back to bf16 for the bank.
        _case(name="stack_read", kind="read", fmt="e4m3", Hq=160, Hkv=160, n_lo=4680, n_hi=4680, past_lo=4703,
              past_hi=4703),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    top = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["attend", "attend", "attend", "attend", "write", "read"])
        c = _case(kind=kind, fmt=rng.choice(["bf16", "e4m3"]), d=rng.choice([128, 128, 64]),
                  page=rng.choice([16, 32, 64, 128, 256]), B=_log(rng, 1, 48), mix=rng.randrange(1 << 20))
        hkv = rng.choice([1, 2, 4, 8, 12, 40])
        group = rng.choice([1, 1, 2, 3, 4, 5, 7, 8]) if kind == "attend" else 1
        c["Hkv"], c["Hq"] = hkv, hkv * group
        chunk = 1 if kind == "attend" and rng.random() < 0.35 else _log(rng, 2, 4680)
        c["n_hi"] = chunk
        c["n_lo"] = rng.choice([chunk, max(1, chunk // 3)])
        c["past_hi"] = _log(rng, 16, 131000) if chunk == 1 else _log(rng, 16, 20000)
        c["past_lo"] = rng.choice([c["past_hi"], c["past_hi"] // 8, 0])
        if kind == "attend":
            c["block"] = rng.choice([1, 1, 1, 0, max(1, chunk // 2), chunk])
            if rng.random() < 0.5:
                c["window"] = _log(rng, 16, 12480)
                c["sinks"] = rng.choice([0, 4, _log(rng, 1, 1560)])
        total = c["B"] * (c["past_hi"] + chunk)
        if total * hkv * c["d"] * 4 < 3e9 and c["B"] * chunk * c["Hq"] * (c["past_hi"] + chunk) < 2.7e9 and _cost(c) <= top:
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


def _visible(c, p, length):
    """[(first, end), ..] of the positions that position p sees."""
    end = length if c["block"] == 0 else min(length, (p // c["block"] + 1) * c["block"])
    if c["window"] == 0:
        return [(0, end)]
    lo, sink = max(0, end - c["window"]), min(c["sinks"], end)
    return [(0, end)] if sink >= lo else [(0, sink), (lo, end)]


def work(c):
    d, row = c["d"], 4 * c["d"] if c["fmt"] == "bf16" else 2 * c["d"] + 2     # a position's key and value in the cache
    if c["kind"] != "attend":
        rows = sum(n for n, _ in _sizes(c)) * c["Hkv"]
        return {"bytes": rows * (4 * d + row), "flops": 0 if c["fmt"] == "bf16" else rows * 4 * d}
    keys = pairs = rows = 0
    for n, length in _sizes(c):
        lo, sink = length, 0
        for p in range(length - n, length):
            v = _visible(c, p, length)
            pairs += sum(e - f for f, e in v)
            lo = min(lo, v[-1][0])
            sink = max(sink, v[0][1] if len(v) > 1 else 0)
        keys += length - lo + min(sink, lo)
        rows += n
    return {"bytes": keys * c["Hkv"] * row + 4 * d * rows * c["Hq"], "flops": 4 * d * pairs * c["Hq"]}


def _cost(c):
    """About the seconds of a pass."""
    w = work(c)
    return w["flops"] / 1e15 + w["bytes"] / 5e12


# ---------------------------------------------------------------- the cache in plain torch
def _quantise(x):
    """e4m3 codes and scale bytes of rows x [.., d]."""
    x = x.float()
    a = x.abs().amax(-1)
    # the smallest e with a <= 448 * 2^e; 448 = 0.875 * 2^9, a = m * 2^q with 0.5 <= m < 1
    m, q = torch.frexp(a)
    e = torch.where(m <= 0.875, q - 9, q - 8)
    e = torch.where(a > 0, e.clamp(min=EMIN), torch.zeros_like(e))
    bad = ~torch.isfinite(a)
    e = torch.where(bad, torch.zeros_like(e), e)
    y = torch.ldexp(x, -e[..., None])
    y = torch.where(bad[..., None], torch.full_like(y, float("nan")), y)
    return y.to(torch.float8_e4m3fn), torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8)


def _scale(byte):
    s = torch.ldexp(torch.ones(byte.shape, device=byte.device), byte.int() - 127)
    return torch.where(byte == 255, torch.full_like(s, float("nan")), s)


def _pooled(codes, scale):
    return codes.float() if scale is None else codes.float() * _scale(scale)[..., None]


def _slots(s):
    """Page and slot of every packed row's position."""
    pos = s["pos"]
    return s["table"][s["seq"], pos // s["case"]["page"]].long(), pos % s["case"]["page"]


def _plain_write(s):
    page, slot = _slots(s)
    for pool, scales, x in ((s["k"], s["ks"], s["kn"]), (s["v"], s["vs"], s["vn"])):
        x = x.transpose(0, 1)                                 # [rows][H][d]
        if scales is None:
            pool[page, :, slot] = x
        else:
            codes, byte = _quantise(x)
            pool.view(torch.uint8)[page, :, slot] = codes.view(torch.uint8)
            scales[page, :, slot] = byte
    return _pool(s)


def _pool(s):
    return {"k": s["k"], "v": s["v"]} if s["ks"] is None else {"k": s["k"], "v": s["v"], "ks": s["ks"], "vs": s["vs"]}


def _plain_read(s):
    page, slot = _slots(s)
    out = {}
    for name, pool, scales in (("k", s["k"], s["ks"]), ("v", s["v"], s["vs"])):
        x = pool.view(torch.uint8)[page, :, slot].view(pool.dtype) if scales is not None else pool[page, :, slot]
        x = _pooled(x, None if scales is None else scales[page, :, slot])
        out[name] = x.to(torch.bfloat16).transpose(0, 1).contiguous()
    return out


def _all_keys(pool, scales, table):
    """[B][H][positions][d] in 32 bits."""
    t = table.long()
    raw = pool.view(torch.uint8)[t].view(pool.dtype) if scales is not None else pool[t]
    x = _pooled(raw, None if scales is None else scales[t])   # [B][pages][H][page][d]
    return x.transpose(1, 2).flatten(2, 3)


def _plain_attend(s):
    c = s["case"]
    B, H, G, d, n = c["B"], c["Hkv"], c["Hq"] // c["Hkv"], c["d"], s["n_max"]
    k, v = _all_keys(s["k"], s["ks"], s["table"]), _all_keys(s["v"], s["vs"], s["table"])
    row = s["row_start"][:-1, None].long() + torch.arange(n, device="cuda")
    used = row < s["row_start"][1:, None]
    row = torch.where(used, row, torch.zeros_like(row))
    q = s["q"][:, row].float().view(H, G, B, n, d).permute(2, 0, 1, 3, 4).reshape(B, H, G * n, d)
    score = (q @ k.transpose(-1, -2)).mul_(1.0 / math.sqrt(d))
    length = s["seq_len"][:, None].long()
    p = length - (s["row_start"][1:] - s["row_start"][:-1])[:, None] + torch.arange(n, device="cuda")
    end = length.expand_as(p) if c["block"] == 0 else torch.minimum(length, (p // c["block"] + 1) * c["block"])
    j = torch.arange(k.shape[2], device="cuda")
    see = j < end[..., None]
    if c["window"]:
        see &= (j >= end[..., None] - c["window"]) | (j < c["sinks"])
    score = score.view(B, H, G, n, -1).masked_fill_(~see[:, None, None], float("-inf"))
    top = score.amax(-1, keepdim=True)
    score = score.sub_(torch.where(torch.isfinite(top), top, torch.zeros_like(top))).exp_()
    total = score.sum(-1, keepdim=True)
    o = score.view(B, H, G * n, -1) @ v
    o = o.view(B, H, G, n, d) / torch.where(total > 0, total, torch.ones_like(total))
    out = torch.empty_like(s["q"])
    out[:, row[used]] = o.permute(1, 2, 0, 3, 4).reshape(c["Hq"], B, n, d)[:, used].to(out.dtype)
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


def prepare(c, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    sizes = _sizes(c)
    T, H, d, page = sum(n for n, _ in sizes), c["Hkv"], c["d"], c["page"]
    pages = [-(-length // page) for _, length in sizes]
    total = sum(pages) + 3                                    # some pages are in nobody's hands
    order = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
    table = torch.zeros(c["B"], max(pages), dtype=torch.int32, device="cuda")
    at = 0
    for b, m in enumerate(pages):
        table[b, :m] = order[at:at + m]
        at += m
    starts = [0]
    for n, _ in sizes:
        starts.append(starts[-1] + n)
    s = {"case": c, "n_max": max(n for n, _ in sizes), "table": table, "ks": None, "vs": None,
         "seq_len": torch.tensor([length for _, length in sizes], dtype=torch.int32, device="cuda"),
         "row_start": torch.tensor(starts, dtype=torch.int32, device="cuda")}
    s["seq"] = torch.repeat_interleave(torch.arange(c["B"], device="cuda"),
                                       torch.tensor([n for n, _ in sizes], device="cuda"))
    first = torch.tensor([length - n for n, length in sizes], device="cuda")
    s["pos"] = first[s["seq"]] + torch.arange(T, device="cuda") - s["row_start"][s["seq"]]
    s["first"] = first.to(torch.int32)
    if c["kind"] == "write":
        empty = torch.zeros(total, H, page, d, dtype=torch.bfloat16, device="cuda")
        s["k"], s["v"] = empty, empty.clone()
        # rows of different magnitudes: a quantised row carries its own scale
        size = torch.exp2(torch.randint(-3, 4, (H, T, 1), generator=gen, device="cuda").float())
        s["kn"] = (_keys(c, gen, T, H).transpose(0, 1) * size).to(torch.bfloat16).contiguous()
        s["vn"] = (torch.randn(H, T, d, generator=gen, device="cuda") * size).to(torch.bfloat16)
    else:
        s["k"] = _keys(c, gen, total, H, page)
        s["v"] = torch.randn(total, H, page, d, generator=gen, device="cuda", dtype=torch.bfloat16)
    if c["fmt"] == "e4m3":
        (s["k"], s["ks"]), (s["v"], s["vs"]) = _quantise(s["k"]), _quantise(s["v"])
    if c["kind"] == "attend":
        s["q"] = _keys(c, gen, T, c["Hq"]).transpose(0, 1).contiguous()
    if own:
        from paper_2608_27922_gb300 import dkv
        s["cache"] = dkv.PagedCache(H, d, page, total, c["fmt"], k=s["k"], v=s["v"], k_scale=s["ks"], v_scale=s["vs"])
        s["seqs"] = dkv.CacheSeqs(table, s["seq_len"], s["row_start"])
    return s


def run(s):
    c = s["case"]
    if c["kind"] == "write":
        if own:
            s["cache"].write(s["kn"], s["vn"], s["seqs"])
            return _pool(s)
        return _plain_write(s)
    if c["kind"] == "read":
        if own:
            k, v = s["cache"].read(s["seqs"], s["first"], s["pos"].numel())
            return {"k": k, "v": v}
        return _plain_read(s)
    if own:
        return {"o": s["cache"].attend(s["q"], s["seqs"], window=c["window"], sinks=c["sinks"], block=c["block"],
                                       max_rows=s["n_max"])}
    return _plain_attend(s)


# ---------------------------------------------------------------- the definition in 64 bits
def _decode(codes, scale):
    """Values of e4m3 codes (sign, 4 exponent bits of bias 7, 3 mantissa bits; 0x7f and 0xff are NaN) times their
    row's scale."""
    b = codes.view(torch.uint8).to(torch.int64)
    e, m = (b >> 3) & 15, (b & 7).double()
    x = torch.where(e > 0, (8 + m) * torch.exp2((e - 10).double()), m * 2.0 ** -9)
    x = torch.where((b & 127) == 127, torch.full_like(x, float("nan")), x) * torch.where(b > 127, -1.0, 1.0)
    s = torch.exp2((scale.to(torch.int64) - 127).double())
    return x * torch.where(scale == 255, torch.full_like(s, float("nan")), s)[..., None]


def exact(c, seed):
    s = prepare(c, seed)
    starts, lens = s["row_start"].tolist(), s["seq_len"].tolist()
    if c["kind"] == "write":
        return _exact_write(s, starts, lens)
    pools = [(s[name], s[name + "s"]) for name in ("k", "v")]

    def rows(pool, b, h, lo, hi):
        """Positions [lo, hi) of sequence b and head h."""
        j = torch.arange(lo, hi, device="cuda")
        page, slot = s["table"][b, j // c["page"]].long(), j % c["page"]
        x, sc = pool
        if sc is None:
            return x[page, h, slot].double()
        return _decode(x.view(torch.uint8)[page, h, slot], sc[page, h, slot])

    if c["kind"] == "read":
        return {name: torch.stack([torch.cat([rows(pool, b, h, lens[b] - (starts[b + 1] - starts[b]), lens[b])
                                              for b in range(c["B"])]) for h in range(c["Hkv"])])
                for name, pool in zip(("k", "v"), pools)}
    if work(c)["flops"] > 4e12:
        return None
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    G = c["Hq"] // c["Hkv"]
    for b in range(c["B"]):
        L, a = lens[b], starts[b]
        for h in range(c["Hkv"]):
            k, v = rows(pools[0], b, h, 0, L), rows(pools[1], b, h, 0, L)
            for i in range(a, starts[b + 1], 512):
                z = min(i + 512, starts[b + 1])
                p = torch.arange(L - starts[b + 1] + i, L - starts[b + 1] + z, device="cuda")
                end = torch.full_like(p, L) if c["block"] == 0 else ((p // c["block"] + 1) * c["block"]).clamp(max=L)
                j = torch.arange(L, device="cuda")[None]
                hide = j >= end[:, None]
                if c["window"]:
                    hide |= (j < end[:, None] - c["window"]) & (j >= c["sinks"])
                for g in range(G):
                    x = (s["q"][h * G + g, i:z].double() @ k.T) / math.sqrt(c["d"])
                    out[h * G + g, i:z] = torch.softmax(x.masked_fill(hide, -math.inf), -1) @ v
    return {"o": out}


def _exact_write(s, starts, lens):
    """The pages with the new rows in them; of a quantised row the values that its codes stand for before they are
    rounded (its scale byte is a whole number)."""
    page = s["case"]["page"]
    at = torch.tensor([lens[b] - starts[b + 1] + r for b in range(s["case"]["B"])
                       for r in range(starts[b], starts[b + 1])], device="cuda")
    p = s["table"][s["seq"], at // page].long()
    out = {}
    for name, new in (("k", s["kn"]), ("v", s["vn"])):
        x, pool = new.double().transpose(0, 1), s[name].double()
        if s[name + "s"] is not None:
            top = x.abs().amax(-1, keepdim=True)
            e = torch.where(top > 0, torch.ceil(torch.log2(top / 448.0)).clamp(min=EMIN), torch.zeros_like(top))
            x = x * torch.exp2(-e)
            out[name + "s"] = None
        pool[p, :, at % page] = x
        out[name] = pool
    return out
