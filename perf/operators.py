"""Operators of a paged cache in 8 bits: what a serving program runs between the prefill and the last token.

The cache holds K and V of every token as 8-bit codes (E4M3 floats or integers) in pages of 32 to 256 tokens,
with one scale for each page, KV head and tensor.  Four operators work on it:

* ``append``  quantises new tokens into the pages of their sequences: whole prompts, pieces, single tokens;
* ``attend``  attention of the newest tokens over their sequences: one token, a few drafted ones, pieces of prompts,
  with capped scores, a bias by distance and a prefix that every token sees;
* ``compact`` gathers the tokens that an eviction kept (other ones for each head) into fewer pages;
* ``fork``    pages change hands: sequences are forked, get pages for their next tokens (a shared last page is
  copied first), and are given up again.

Head shapes are those of the benchmark configurations (8 KV heads x 4 query heads, head_dim 128) and their
neighbours, lengths run from one token to 128 Ki.  Plans, tables and pools are what a program keeps.

A page of one head, P tokens, is [P, 128] bytes for K and for V.
"""
import math
import random

import torch

D = 128
own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
TINY = 2.0 ** -126


# ------------------------------------------------------------------ cases

def _append(name, dtype, fmt, batch, heads, page, old, new, mix=1, positions=False):
    c = dict(kind="append", dtype=dtype, fmt=fmt, batch=batch, heads=heads, page=page, old_lo=old[0], old_hi=old[1],
             new_lo=new[0], new_hi=new[1], mix=mix, positions=positions)
    return dict(c, name=name) if name else c


def _attend(name, dtype, fmt, batch, heads, group, page, length, new, mix=1, positions=False, softcap=0.0, slopes=False,
            prefix=False, lse=False):
    c = dict(kind="attend", dtype=dtype, fmt=fmt, batch=batch, heads=heads, group=group, page=page, len_lo=length[0],
             len_hi=length[1], new_lo=new[0], new_hi=new[1], mix=mix, positions=positions, softcap=softcap,
             slopes=slopes, prefix=prefix, lse=lse)
    return dict(c, name=name) if name else c


def _compact(name, fmt, batch, heads, page, length, kept, mix=1):
    c = dict(kind="compact", fmt=fmt, batch=batch, heads=heads, page=page, len_lo=length[0], len_hi=length[1],
             kept=kept, mix=mix)
    return dict(c, name=name) if name else c


def _fork(name, fmt, heads, page, seqs, beams, length, grow, mix=1):
    c = dict(kind="fork", fmt=fmt, heads=heads, page=page, seqs=seqs, beams=beams, len_lo=length[0], len_hi=length[1],
             grow=grow, mix=mix)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the prompt of the 32k-context configuration is stored: one layer, K and V
        _append("append_prompt_32k", "f16", "e4m3", 1, 8, 64, (0, 0), (32768, 32768)),
        # one decode step of a full batch: a token a sequence, pages begun and half full
        _append("append_step_64", "bf16", "i8", 64, 8, 64, (100, 8000), (1, 1), mix=2),
        # pieces of several prompts behind what is there, single precision, with positions
        _append("append_pieces", "f32", "e4m3", 12, 8, 128, (1, 3000), (3, 900), mix=3, positions=True),
        # the smallest step: one sequence, a short context, one token
        _attend("attend_one_short", "f16", "e4m3", 1, 8, 4, 64, (700, 700), (1, 1)),
        # a decode step of a batch of ragged contexts
        _attend("attend_step_32", "bf16", "i8", 32, 8, 4, 32, (150, 8192), (1, 1), mix=4),
        # a decode step over a very long context
        _attend("attend_step_128k", "f16", "e4m3", 1, 8, 4, 128, (131071, 131071), (1, 1), lse=True),
        # drafted tokens checked over an evicted context (positions have gaps), capped scores and a bias by distance
        _attend("attend_draft", "f32", "i8", 6, 8, 4, 64, (1000, 2055), (4, 8), mix=5, positions=True, softcap=30.0,
                slopes=True, lse=True),
        # a piece of a long prompt over what is stored
        _attend("attend_piece_2k", "bf16", "e4m3", 1, 8, 4, 64, (16384, 16384), (2048, 2048)),
        # short prompts of a batch with prefixes that every token sees, capped scores, one query head per KV head
        _attend("attend_prompts", "f16", "i8", 5, 16, 1, 64, (200, 1500), (200, 1500), mix=6, softcap=50.0, prefix=True),
        # an eviction at 32k keeps 2048 tokens of each head
        _compact("compact_32k", "e4m3", 1, 8, 64, (32768, 32768), 2048),
        # forked beams of one short sequence
        _fork("fork_small", "i8", 8, 32, 1, 4, (333, 333), 1),
        # a batch forks its long sequences and every branch gets room for drafted tokens
        _fork("fork_batch", "e4m3", 8, 64, 24, 4, (500, 9000), 6, mix=7),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "attend", "compact", "fork"])
    dtype, fmt = rng.choice(["f16", "bf16", "f16", "bf16", "f32"]), rng.choice(["e4m3", "i8"])
    page, mix = rng.choice([32, 64, 64, 128, 256]), rng.randrange(1 << 20)
    heads = rng.choice([1, 2, 4, 8, 8, 16])
    if kind == "append":
        batch = _log(rng, 1, 64)
        top = _log(rng, 1, max(1, 32768 * 7 // (heads * batch * (2 if dtype == "f32" else 1))))
        old = _log(rng, 1, 4000)
        return _append(None, dtype, fmt, batch, heads, page, (rng.randrange(old + 1), old), (max(1, top // 5), top), mix,
                       rng.random() < 0.5)
    if kind == "attend":
        batch = _log(rng, 1, 48)
        group = rng.choice([1, 2, 4, 4, 5, 8])
        room = 131071 * 8 // (heads * batch * max(group, 2))
        new = rng.choice([1, 1, _log(rng, 2, 16), _log(rng, 17, 2048)])
        new = min(new, max(1, (1 << 17) // (batch * heads * group)))
        length = _log(rng, new + 40, max(new + 41, min(room, (1 << 28) // (new * batch * heads * group))))
        return _attend(None, dtype, fmt, batch, heads, group, page, (max(new, length // 12), length),
                       (max(1, new // 3), new), mix, rng.random() < 0.3, rng.choice([0.0, 0.0, 20.0, 50.0]),
                       rng.random() < 0.3, rng.random() < 0.3, rng.random() < 0.5)
    if kind == "compact":
        batch = _log(rng, 1, 16)
        length = _log(rng, 64, max(65, 32768 * 8 // (heads * batch)))
        return _compact(None, fmt, batch, heads, page, (max(48, length // 3), length), _log(rng, 16, max(17, length // 3)), mix)
    seqs, beams = _log(rng, 1, 24), rng.choice([1, 2, 3, 4, 6])
    length = _log(rng, 20, min(9000, 200000 * 8 // (heads * seqs * beams)))
    return _fork(None, fmt, heads, page, seqs, beams, (max(1, length // 10), length), rng.choice([1, 1, 2, 6, 40]), mix)


# ------------------------------------------------------------------ sizes of a case, from the case alone

def _ragged(lo, hi, n, mix):
    """n lengths spread over lo..hi, the longest first."""
    rng = random.Random(mix)
    return [hi] + [_log(rng, max(lo, 1), hi) if hi > 0 else 0 for _ in range(n - 1)]


def _sizes(c):
    """(tokens in the cache before the call or in all, new tokens) of each sequence."""
    if c["kind"] == "append":
        return _ragged(c["old_lo"], c["old_hi"], c["batch"], c["mix"]), _ragged(c["new_lo"], c["new_hi"], c["batch"], c["mix"] + 1)
    if c["kind"] == "attend":
        lens = _ragged(c["len_lo"], c["len_hi"], c["batch"], c["mix"])
        return lens, [min(n, m) for n, m in zip(lens, _ragged(c["new_lo"], c["new_hi"], c["batch"], c["mix"] + 1))]
    if c["kind"] == "compact":
        lens = _ragged(c["len_lo"], c["len_hi"], c["batch"], c["mix"])
        return lens, [min(n, c["kept"]) for n in lens]
    return _ragged(c["len_lo"], c["len_hi"], c["seqs"], c["mix"]), [c["grow"]] * (c["seqs"] * c["beams"])


def _pages(tokens, page):
    return -(-tokens // page)


def _prefixes(c, lens):
    return [n // 3 for n in lens]


def _copied(c):
    """Sequences whose branches all get a copy of their last page."""
    return sum(n % c["page"] != 0 for n in _sizes(c)[0])


def work(case):
    c, page, heads = case, case["page"], case["heads"]
    lens, new = _sizes(c)
    if c["kind"] == "append":
        elt = 4 if c["dtype"] == "f32" else 2
        rows = sum(new) * heads
        scales = sum(_pages(n + m, page) - n // page for n, m in zip(lens, new)) * heads * 8
        return {"bytes": rows * 2 * D * (elt + 1) + scales + (rows * 4 if c["positions"] else 0), "flops": rows * 2 * D * 3}
    if c["kind"] == "attend":
        elt = 4 if c["dtype"] == "f32" else 2
        hq = heads * c["group"]
        seen = 0
        for n, m, p in zip(lens, new, _prefixes(c, lens)):
            at = [n - m + i + 1 for i in range(m)]
            seen += sum(max(x, p) for x in at) if c["prefix"] else sum(at)
        kv = sum(lens) * heads * (2 * D + (4 if c["positions"] else 0)) + sum(_pages(n, page) for n in lens) * (heads * 8 + 4)
        return {"bytes": kv + 2 * sum(new) * hq * D * elt + (sum(new) * hq * 4 if c["lse"] else 0), "flops": 4 * D * hq * seen}
    if c["kind"] == "compact":
        rows = sum(new) * heads
        return {"bytes": rows * (2 * 2 * D + 2 * 4 + 4), "flops": rows * 2 * D * 3}
    held = sum(_pages(n, page) for n in lens) * c["beams"]
    moved = _copied(c) * c["beams"] * 2 * heads * (2 * D * page + 8)
    return {"bytes": held * (4 + 4 + 8 + 4 + 8) + 4 * _pool_pages(c) + moved, "flops": held * 2}


# ------------------------------------------------------------------ the definition of the codes, in torch

def _scale(amax, fmt):
    """The scale of a page whose largest finite magnitude is amax (f32)."""
    if fmt == "i8":
        return (amax.double() / 127).float().clamp_min(TINY)
    m, e = torch.frexp(amax)                                       # amax = m 2^e, m in [0.5, 1); 448 = 0.875 2^9
    e = torch.where(m <= 0.875, e - 9, e - 8)
    return ((e.clamp(-126, 127) + 127) << 23).view(torch.float32).masked_fill(amax == 0, TINY)


def _codes(x, s, fmt):
    """The codes of the values x at the scale s: nearest, ties to even; what is too large saturates, NaN is zero."""
    x = torch.nan_to_num(x.double(), nan=0.0) / s.double()
    if fmt == "i8":
        return torch.round(x.clamp(-127, 127)).to(torch.int8)
    return x.clamp(-448, 448).float().to(torch.float8_e4m3fn)


def _amax(x):
    """Largest finite magnitude over the last two dimensions, kept."""
    a = x.abs()
    return torch.where(torch.isfinite(a), a, 0.0).amax(dim=(-2, -1), keepdim=True)


def _typed(pool, fmt):
    return pool.view(torch.int8 if fmt == "i8" else torch.float8_e4m3fn)


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _tokens(g, rows, heads):
    """Rows like those of a cache: a mean of its own for each head's dimension, a few heavy tokens."""
    x = _normal(g, rows, heads, D) + 0.7 * _normal(g, 1, heads, D)
    heavy = 1 + 3 * (torch.rand(rows, 1, 1, generator=g, device="cuda") < 0.05).float()
    return x * heavy


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _table(g, counts, width, n_pages, begin=0):
    """A block table whose sequences' pages lie scattered over the pool; unused entries are -1."""
    order = begin + torch.randperm(n_pages - begin, generator=g, device="cuda").to(torch.int32)
    at = torch.arange(width, device="cuda")[None, :]
    n = torch.tensor(counts, device="cuda")[:, None]
    start = torch.cumsum(n, 0) - n
    return torch.where(at < n, order[(start + at).clamp_max(n_pages - begin - 1)], -1).to(torch.int32).contiguous()


class _Cache:
    """What ``binding.new_cache`` makes: the pools of one layer."""

    def __init__(self, n_pages, heads, page, fmt, positions):
        self.k, self.v = (torch.zeros(n_pages, heads, page, D, dtype=torch.uint8, device="cuda") for _ in range(2))
        self.k_scale, self.v_scale = (torch.zeros(n_pages, heads, device="cuda") for _ in range(2))
        self.pos = torch.zeros(n_pages, heads, page, dtype=torch.int32, device="cuda") if positions else None
        self.page, self.fmt, self.heads, self.n_pages = page, fmt, heads, n_pages

    def handle(self):
        from paper_2507_06517_amd import binding as sb
        return sb.Cache(self.k, self.v, self.k_scale, self.v_scale, self.pos, self.page, self.fmt)

    def outputs(self):
        o = dict(k=_typed(self.k, self.fmt), v=_typed(self.v, self.fmt), k_scale=self.k_scale, v_scale=self.v_scale)
        return dict(o, pos=self.pos) if self.pos is not None else o


def _fill(cache, g, table, lens, gaps=False):
    """Stores `lens` tokens of each sequence, as append() would have."""
    page, heads = cache.page, cache.heads
    for b, n in enumerate(lens):
        m = _pages(n, page)
        if not m:
            continue
        ids = table[b, :m].long()
        for pool, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
            x = torch.zeros(m * page, heads, D, device="cuda")
            x[:n] = _tokens(g, n, heads)
            x = x.reshape(m, page, heads, D).transpose(1, 2).contiguous()
            s = _scale(_amax(x), cache.fmt)
            pool[ids] = _codes(x, s, cache.fmt).view(torch.uint8)
            scale[ids] = s[..., 0, 0]
        if cache.pos is not None:
            step = torch.randint(1, 4 if gaps else 2, (heads, m * page), generator=g, device="cuda", dtype=torch.int32)
            p = torch.cumsum(step, 1, dtype=torch.int32) - step[:, :1]
            cache.pos[ids] = p.reshape(heads, m, page).transpose(0, 1)


def _starts(new):
    out = [0]
    for n in new:
        out.append(out[-1] + n)
    return out


def _pool_pages(c):
    lens, new = _sizes(c)
    if c["kind"] == "append":
        return sum(_pages(n + m, c["page"]) for n, m in zip(lens, new)) + 3
    if c["kind"] == "attend":
        return sum(_pages(n, c["page"]) for n in lens) + 3
    if c["kind"] == "compact":
        return sum(_pages(n, c["page"]) + _pages(m, c["page"]) for n, m in zip(lens, new)) + 3
    more = [c["beams"] * (_pages(n + c["grow"], c["page"]) - n // c["page"]) for n in lens]
    return sum(_pages(n, c["page"]) for n in lens) + sum(more) + 3


def prepare(case, seed):
    c, g = case, _gen(seed)
    page, heads, n_pages = c["page"], c["heads"], _pool_pages(case)
    lens, new = _sizes(c)
    positions = c["kind"] == "compact" or bool(c.get("positions"))
    cache = _Cache(n_pages, heads, page, c["fmt"], positions)
    s = dict(case=c, cache=cache, lens=_ints(lens), new=_ints(new), max_new=max(new))
    if c["kind"] == "append":
        counts = [_pages(n + m, page) for n, m in zip(lens, new)]
        s["table"] = _table(g, counts, max(counts), n_pages)
        _fill(cache, g, s["table"], lens)
        dt = DTYPES[c["dtype"]]
        s["K"], s["V"] = (_tokens(g, sum(new), heads).to(dt) for _ in range(2))
        s["cu"] = _ints(_starts(new))
        s["positions"] = None
        if positions:
            s["positions"] = torch.cat([torch.arange(n, n + m, dtype=torch.int32, device="cuda") for n, m in zip(lens, new)])
    elif c["kind"] == "attend":
        counts = [_pages(n, page) for n in lens]
        s["table"] = _table(g, counts, max(counts), n_pages)
        _fill(cache, g, s["table"], lens, gaps=True)
        hq = heads * c["group"]
        s["Q"] = (1.5 * _normal(g, sum(new), hq, D)).to(DTYPES[c["dtype"]])
        s["cu"] = _ints(_starts(new))
        s["slopes"] = torch.pow(2.0, -8.0 * torch.arange(1, hq + 1, device="cuda") / hq).float() if c["slopes"] else None
        s["prefix"] = _ints(_prefixes(c, lens)) if c["prefix"] else None
        # the newest tokens' own positions: behind every kept one where the context has gaps
        s["q_pos"] = None
        if positions:
            s["q_pos"] = torch.cat([torch.arange(3 * n, 3 * n + m, dtype=torch.int32, device="cuda") for n, m in zip(lens, new)])
    elif c["kind"] == "compact":
        counts = [_pages(n, page) for n in lens]
        half = sum(counts)
        s["table"] = _table(g, counts, max(counts), half)
        s["table_out"] = _table(g, [_pages(m, page) for m in new], _pages(max(new), page), n_pages, half)
        _fill(cache, g, s["table"], lens)
        kept = torch.full((c["batch"], heads, max(new)), -1, dtype=torch.int32, device="cuda")
        for b, (n, m) in enumerate(zip(lens, new)):                # what an eviction keeps: scores' best, the last ones always
            score = torch.rand(heads, n, generator=g, device="cuda")
            score[:, max(0, n - 32):] += 1
            kept[b, :, :m] = score.topk(m, dim=1).indices.sort(dim=1).values.to(torch.int32)
        s["kept"] = kept
    else:
        counts = [_pages(n, page) for n in lens]
        rows = c["seqs"] * c["beams"]
        width = max(_pages(n + c["grow"], page) for n in lens)
        s["table"] = _table(g, counts, width, n_pages)
        _fill(cache, g, s["table"], lens)
        s["refs"] = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
        held = s["table"][s["table"] >= 0].long()
        s["refs"][held] = 1
        parent = torch.arange(c["seqs"], device="cuda").repeat_interleave(c["beams"])
        s["parent"] = parent[torch.randperm(rows, generator=g, device="cuda")].to(torch.int32)
    return s


# ------------------------------------------------------------------ one pass

def run(state):
    return {"append": _run_append, "attend": _run_attend, "compact": _run_compact, "fork": _run_fork}[state["case"]["kind"]](state)


def _write(pool, scale, ids, live, codes, s):
    pool[ids[live]] = codes.view(torch.uint8)[live]
    scale[ids[live]] = s[..., 0, 0][live]


def _run_append(s):
    cache = s["cache"]
    if own:
        from paper_2507_06517_amd import binding as sb
        sb.cache_append(cache.handle(), s["table"], s["lens"], s["K"], s["V"], cu_new=s["cu"], max_new=s["max_new"],
                        positions=s["positions"])
        return cache.outputs()
    page, fmt = cache.page, cache.fmt
    n, m, cu = s["lens"].long()[:, None], s["new"].long()[:, None], s["cu"].long()[:-1, None]
    j = n // page + torch.arange((s["max_new"] + page - 2) // page + 1, device="cuda")     # the pages that get tokens
    live = j * page < n + m
    ids = torch.gather(s["table"].long(), 1, j.clamp_max(s["table"].shape[1] - 1)).clamp_min(0)
    slot = j[..., None] * page + torch.arange(page, device="cuda")                         # [B, T, P]
    before, fresh = slot < n[..., None], (slot >= n[..., None]) & (slot < (n + m)[..., None])
    row = torch.where(fresh, cu[..., None] + slot - n[..., None], 0)
    before, fresh = before[:, :, None, :, None], fresh[:, :, None, :, None]
    for x, pool, scale in ((s["K"], cache.k, cache.k_scale), (s["V"], cache.v, cache.v_scale)):
        x = torch.where(fresh, x[row].transpose(2, 3).float(), 0.0)                        # [B, T, H, P, D]
        codes = _typed(pool[ids], fmt)
        had = scale[ids][..., None, None]
        to = torch.maximum(_scale(_amax(x), fmt), torch.where(before.any(dim=3, keepdim=True), had, 0.0))
        old = torch.where(before, codes.double() * had.double(), 0.0)
        _write(pool, scale, ids, live, _codes(torch.where(fresh, x.double(), old), to, fmt), to)
    if cache.pos is not None:
        at = (ids[..., None].expand_as(slot)[fresh[:, :, 0, :, 0]], (slot % page)[fresh[:, :, 0, :, 0]])
        cache.pos[at[0], :, at[1]] = s["positions"][row[fresh[:, :, 0, :, 0]]][:, None]
    return cache.outputs()


def _dequantised(cache, table, dtype):
    """K and V of every sequence, [B, H, tokens of the table's pages, D]; pages that a sequence lacks repeat page 0."""
    ids = table.long().clamp_min(0)
    out = []
    for pool, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        x = _typed(pool[ids], cache.fmt).to(dtype) * scale[ids][..., None, None].to(dtype)
        out.append(x.transpose(1, 2).reshape(ids.shape[0], cache.heads, -1, D))
    return out


def _run_attend(s):
    c, cache = s["case"], s["cache"]
    if own:
        from paper_2507_06517_amd import binding as sb
        return sb.cache_attend(cache.handle(), s["table"], s["lens"], s["Q"], c["group"], cu_q=s["cu"], max_q=s["max_new"],
                               softcap=c["softcap"], slopes=s["slopes"], prefix=s["prefix"], q_pos=s["q_pos"],
                               want_lse=c["lse"])
    B, H, G = c["batch"], c["heads"], c["group"]
    K, V = _dequantised(cache, s["table"], torch.float32)
    L, M, total = K.shape[2], s["max_new"], s["Q"].shape[0]
    cu, n = s["cu"].long(), s["lens"].long()
    i = torch.arange(M, device="cuda")
    row = (cu[:-1, None] + i).clamp_max(total - 1)                                          # [B, M]
    Q = s["Q"][row].float().reshape(B, M, H, G, D).permute(0, 2, 3, 1, 4).reshape(B, H, G * M, D)
    S = torch.matmul(Q, K.transpose(2, 3)).reshape(B, H, G, M, L) / math.sqrt(D)
    if c["softcap"]:
        S = c["softcap"] * torch.tanh(S / c["softcap"])
    slot = torch.arange(L, device="cuda")
    q_slot = (n - (cu[1:] - cu[:-1]))[:, None] + i                                          # [B, M]
    if c["slopes"]:
        k_at = slot[None, None, :].float()
        q_at = q_slot[:, None, None, :, None].float()
        if cache.pos is not None:
            k_at = cache.pos[s["table"].long().clamp_min(0)].transpose(1, 2).reshape(B, H, L).float()
            q_at = s["q_pos"][row][:, None, None, :, None].float()
        S = S - s["slopes"].reshape(H, G, 1, 1) * (q_at - k_at[:, :, None, None, :]).abs()
    seen = slot <= q_slot[..., None]
    if s["prefix"] is not None:
        seen = seen | (slot < s["prefix"].long()[:, None, None])
    seen = (seen & (slot < n[:, None, None]))[:, None, None]
    S = S.masked_fill(~seen, -math.inf)
    top = S.amax(dim=-1, keepdim=True)
    P = torch.exp(S - torch.where(top.isfinite(), top, 0.0))
    total_p = P.sum(dim=-1, keepdim=True)
    O = torch.matmul(P.reshape(B, H, G * M, L), V).reshape(B, H, G, M, D) / total_p
    at = torch.arange(total, device="cuda")
    b = torch.searchsorted(cu[1:].contiguous(), at, right=True)
    out = O.permute(0, 3, 1, 2, 4)[b, at - cu[b]].reshape(total, H * G, D).to(s["Q"].dtype)
    if not c["lse"]:
        return out
    lse = (top + torch.log(total_p))[..., 0].permute(0, 3, 1, 2)[b, at - cu[b]].reshape(total, H * G)
    return out, lse


def _run_compact(s):
    cache = s["cache"]
    if own:
        from paper_2507_06517_amd import binding as sb
        sb.cache_compact(cache.handle(), s["table"], s["lens"], s["kept"], s["new"], s["table_out"])
        return cache.outputs()
    page, fmt, H = cache.page, cache.fmt, cache.heads
    B, width = s["table_out"].shape
    at = torch.arange(width * page, device="cuda")
    kept = torch.nn.functional.pad(s["kept"].long(), (0, width * page - s["kept"].shape[2]), value=-1)
    live = (at < s["new"].long()[:, None])[:, None] & (kept >= 0)                           # [B, H, S]
    kept = kept.clamp_min(0)
    ids = torch.gather(s["table"].long().clamp_min(0)[:, None].expand(B, H, -1), 2, kept // page)
    head, slot = torch.arange(H, device="cuda")[:, None], kept % page
    to = s["table_out"].long()
    there = to >= 0
    fold = lambda x: x.reshape(B, H, width, page, *x.shape[3:]).transpose(1, 2)            # noqa: E731
    for pool, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        x = _typed(pool[ids, head, slot], fmt).double() * scale[ids, head][..., None].double()
        x = fold(torch.where(live[..., None], x, 0.0))                                      # [B, W, H, P, D]
        size = _scale(_amax(x).float(), fmt)
        _write(pool, scale, to, there, _codes(x, size, fmt), size)
    where = torch.where(live, cache.pos[ids, head, slot], -1)
    cache.pos[to[there]] = fold(where)[there]
    return cache.outputs()


def _run_fork(s):
    c, cache = s["case"], s["cache"]
    if own:
        from paper_2507_06517_amd import binding as sb
        handle = cache.handle()
        table, lens = sb.pages_share(s["refs"], s["table"], s["lens"], s["parent"], cache.page)
        longer, copies, status = sb.pages_reserve(s["refs"], table, lens, s["new"], cache.page)
        sb.cache_copy(handle, copies)
        sb.pages_release(s["refs"], table, longer, cache.page)
        return dict(cache.outputs(), table=table, lens=longer, copies=copies, status=status, refs=s["refs"])
    page, refs = cache.page, s["refs"]
    count = lambda x: (x + page - 1) // page                                                # noqa: E731
    # branches hold the pages of the sequence that they come from
    parent = s["parent"].long()
    table, lens = s["table"][parent], s["lens"][parent].long()
    rows, width = table.shape
    at = torch.arange(width, device="cuda")
    held = at < count(lens)[:, None]
    table = torch.where(held, table, -1)
    refs.index_add_(0, table.clamp_min(0).flatten().long(), held.flatten().to(torch.int32))
    # pages for the next tokens: the free page of the lowest number first; a shared last page is replaced by a copy
    grow = s["new"].long()
    last = torch.gather(table.long(), 1, (count(lens) - 1).clamp_min(0)[:, None])[:, 0]
    partial = (grow > 0) & (lens % page != 0)
    same = (last[:, None] == last) & partial[:, None] & partial
    rank = (same & (torch.arange(rows, device="cuda")[:, None] > torch.arange(rows, device="cuda"))).sum(1)
    moves = partial & (rank < refs[last.clamp_min(0)] - 1)
    need = count(lens + grow) - count(lens) + moves
    begin = torch.cumsum(need, 0) - need
    free = torch.sort((refs != 0).to(torch.int32), stable=True).indices                     # free ones first, in order
    lacking = (need.sum() - (refs == 0).sum()).clamp_min(0)
    narrow = (count(lens + grow) > width).sum()
    fine = (lacking == 0) & (narrow == 0)
    first = count(lens) - moves.long()                                                      # the first entry that changes
    k = at - first[:, None]
    takes = (k >= 0) & (k < need[:, None]) & fine
    page_of = free[(begin[:, None] + k).clamp(0, refs.shape[0] - 1)]
    copies = torch.where((moves & fine)[:, None], torch.stack([last, free[begin.clamp_max(refs.shape[0] - 1)]], 1), -1).to(torch.int32)
    refs.index_add_(0, last.clamp_min(0), -(moves & fine).to(torch.int32))
    table = torch.where(takes, page_of.to(torch.int32), table)
    refs.index_add_(0, page_of.flatten(), takes.flatten().to(torch.int32))
    longer = torch.where(fine, lens + grow, lens).to(torch.int32)
    status = torch.stack([lacking, narrow]).to(torch.int32)
    # the copies' contents
    src, dst = (x[copies[:, 0] >= 0] for x in copies.long().unbind(1))
    for pool in (cache.k, cache.v, cache.k_scale, cache.v_scale):
        pool[dst] = pool[src]
    # the branches are given up
    held = at < count(longer.long())[:, None]
    refs.index_add_(0, table.clamp_min(0).flatten().long(), -held.flatten().to(torch.int32))
    return dict(cache.outputs(), table=table, lens=longer, copies=copies, status=status, refs=refs)


# ------------------------------------------------------------------ the definition in 64 bits, sequence by sequence

def _round_e4m3(x):
    """Nearest number of 1 sign, 4 exponent and 3 mantissa bits (least exponent -6, largest 448), ties to even, in doubles."""
    _, e = torch.frexp(x)
    step = ((e.long() - 1).clamp_min(-6) - 3 + 1023 << 52).view(torch.float64)
    return (torch.round(x / step) * step).clamp(-448, 448)


def _scale64(a, fmt):
    a = float(a)
    if fmt == "i8":
        return max(float(torch.tensor(a / 127, dtype=torch.float64).float()), TINY)
    e = -126
    while 448.0 * 2.0 ** e < a:
        e += 1
    return 2.0 ** e


def _exact_cache(cache):
    o = {n: _typed(getattr(cache, n), cache.fmt).double() for n in ("k", "v")}
    o.update(k_scale=cache.k_scale.double(), v_scale=cache.v_scale.double())
    return dict(o, pos=cache.pos.clone()) if cache.pos is not None else o


def _whole(o, fmt):
    return dict(o, k=o["k"].to(torch.int8), v=o["v"].to(torch.int8)) if fmt == "i8" else o


def _nearest(x, fmt):
    return torch.round(x.clamp(-127, 127)) if fmt == "i8" else _round_e4m3(x)


def exact(case, seed):
    s = prepare(case, seed)
    c, cache, page, fmt = case, s["cache"], case["page"], case["fmt"]
    lens, new = _sizes(c)
    table = s["table"].tolist()
    if c["kind"] == "append":
        if sum(_pages(n + m, page) - n // page for n, m in zip(lens, new)) * c["heads"] > 6000:
            return None                                            # page by page here: too long
        o, cu = _exact_cache(cache), s["cu"].tolist()
        for b, (n, m) in enumerate(zip(lens, new)):
            for j in range(n // page, _pages(n + m, page)):
                lo, hi, id_ = max(n, j * page), min(n + m, (j + 1) * page), table[b][j]
                at, row = slice(lo - j * page, hi - j * page), slice(cu[b] + lo - n, cu[b] + hi - n)
                for x, name in ((s["K"], "k"), (s["V"], "v")):
                    fresh = x[row].double()
                    size = fresh.abs().amax(dim=(0, 2)).tolist()
                    for h in range(c["heads"]):
                        to, values = _scale64(size[h], fmt), torch.zeros(page, D, dtype=torch.float64, device="cuda")
                        if lo > j * page:
                            had = float(o[name + "_scale"][id_, h])
                            to = max(to, had)
                            values[:at.start] = _typed(getattr(cache, name)[id_, h], fmt)[:at.start].double() * had
                        values[at] = fresh[:, h]
                        o[name][id_, h] = _nearest(values / to, fmt)
                        o[name + "_scale"][id_, h] = to
                if cache.pos is not None:
                    o["pos"][id_, :, at] = s["positions"][row]
        return _whole(o, fmt)
    if c["kind"] == "attend":
        G, cu = c["group"], s["cu"].tolist()
        out = torch.zeros(s["Q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.zeros(s["Q"].shape[:2], dtype=torch.float64, device="cuda")
        for b, (n, m) in enumerate(zip(lens, new)):
            ids = torch.tensor(table[b][: _pages(n, page)], device="cuda")
            q_slot = torch.arange(n - m, n, device="cuda")
            k_slot = torch.arange(n, device="cuda")
            seen = k_slot[None] <= q_slot[:, None]
            if c["prefix"]:
                seen = seen | (k_slot < _prefixes(c, lens)[b])
            K, V = _dequantised(cache, s["table"][b: b + 1, : len(ids)], torch.float64)
            for h in range(c["heads"]):
                q = s["Q"][cu[b]: cu[b + 1], h * G: (h + 1) * G].double().transpose(0, 1)    # [G, m, D]
                S = q @ K[0, h, :n].t().contiguous() / math.sqrt(D)
                if c["softcap"]:
                    S = torch.tanh(S / c["softcap"]) * c["softcap"]
                if c["slopes"]:
                    k_at, q_at = k_slot.double(), q_slot.double()
                    if cache.pos is not None:
                        k_at, q_at = cache.pos[ids, h].flatten()[:n].double(), s["q_pos"][cu[b]: cu[b + 1]].double()
                    S = S - s["slopes"][h * G: (h + 1) * G, None, None].double() * (q_at[:, None] - k_at).abs()
                S = torch.where(seen, S, -math.inf)
                out[cu[b]: cu[b + 1], h * G: (h + 1) * G] = (torch.softmax(S, -1) @ V[0, h, :n]).transpose(0, 1)
                lse[cu[b]: cu[b + 1], h * G: (h + 1) * G] = torch.logsumexp(S, -1).t()
        return (out, lse) if c["lse"] else out
    if c["kind"] == "compact":
        if sum(_pages(m, page) for m in new) * c["heads"] > 3000:
            return None
        o, kept, to_table = _exact_cache(cache), s["kept"], s["table_out"].tolist()
        for b, m in enumerate(new):
            ids = torch.tensor(table[b][: _pages(lens[b], page)], device="cuda")
            for h in range(c["heads"]):
                for name in ("k", "v"):
                    rows = _typed(getattr(cache, name)[ids, h], fmt).double()
                    rows = (rows * getattr(cache, name + "_scale")[ids, h].double()[:, None, None]).reshape(-1, D)
                    x = torch.zeros(_pages(m, page) * page, D, dtype=torch.float64, device="cuda")
                    x[:m] = rows[kept[b, h, :m].long()]
                    for j in range(_pages(m, page)):
                        part = x[j * page: (j + 1) * page]
                        to = _scale64(part.abs().amax().float(), fmt)
                        o[name][to_table[b][j], h] = _nearest(part / to, fmt)
                        o[name + "_scale"][to_table[b][j], h] = to
                where = torch.full((_pages(m, page) * page,), -1, dtype=torch.int32, device="cuda")
                where[:m] = cache.pos[ids, h].flatten()[kept[b, h, :m].long()]
                o["pos"][torch.tensor(to_table[b][: _pages(m, page)], device="cuda"), h] = where.reshape(-1, page)
        return _whole(o, fmt)
    # fork: the steps one after the other, as a program on the host would do them
    refs, parent = s["refs"].tolist(), s["parent"].tolist()
    rows, sizes = [list(table[p]) for p in parent], [lens[p] for p in parent]
    o = _exact_cache(cache)
    for r, n in zip(rows, sizes):
        for p in r[: _pages(n, page)]:
            refs[p] += 1
    copies = []
    for r, n, m in zip(rows, sizes, new):
        pair = [-1, -1]
        if m and n % page and refs[r[n // page]] > 1:
            p = refs.index(0)
            pair = [r[n // page], p]
            refs[pair[0]] -= 1
            refs[p], r[n // page] = 1, p
        for j in range(_pages(n, page), _pages(n + m, page)):
            r[j] = refs.index(0)
            refs[r[j]] = 1
        copies.append(pair)
    for p, q in copies:
        if p >= 0:
            for name in ("k", "v", "k_scale", "v_scale"):
                o[name][q] = o[name][p]
    longer = [n + m for n, m in zip(sizes, new)]
    for r, n in zip(rows, longer):
        for p in r[: _pages(n, page)]:
            refs[p] -= 1
    return dict(_whole(o, fmt), table=_ints(rows), lens=_ints(longer), copies=_ints(copies), status=_ints([0, 0]), refs=_ints(refs))
