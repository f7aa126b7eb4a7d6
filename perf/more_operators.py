"""More operators of the paged cache as they are timed and checked: pages dealt to the sequences of a batch on the device, pages
of 8-bit codes with a scale for each block of tokens and head, attention of rows over states of another length.

A batch lies in a pool as in perf/operators.py: `table` [seqs, pages of the longest] names the pages of a sequence in a pool
[pages, key-value heads, tokens a page, d]; rows start[s] to start[s + 1] - 1 of the row tensors [rows, heads, d] are those of
sequence s.

`run()` computes a case with elementary torch operations, or, where `own` is set, with the library's calls.  `listed()` holds
the fixed cases, `draw()` gives further ones of the same ranges, `exact()` the results in 64 bits.

Fields of a case: op
  assign  sequences are cut or ended and grow by new rows; pages come from and go back to a stack; tells lengths, row numbers,
          and of every row its position and its place in the pool: `seqs` of them with shortest to longest tokens, of which one in
          `ends` ends and is followed by another of 1 to `prompt` new rows, the others take `new` rows; `pad` rows too many;
          `scarce`: the pool has fewer free pages than asked for
  store   rows written to pages in blocks, and the sequences' last `back` tokens read back
  attend  causal attention of sequences' last rows over pages in blocks
  cross   attention of rows over all of another sequence's states
and form of the pages (plain: the rows' type; fp8, int8: a scale a token and head; fp8_blocks, int8_blocks: a scale for each
`block` tokens and head), dtype of the rows, h / hq key-value and query heads, d head dimension, page tokens a page, seqs
sequences of `new` new rows each (0: all of their tokens), with shortest to longest tokens, `none` of them with no tokens at
all; lse: the logarithm of the softmax sums is returned too; lens: draws the lengths.
"""
import itertools
import math
import random

import torch

own = False

DEV = "cuda"
DEFAULTS = dict(form="plain", dtype="bf16", h=8, hq=32, d=128, page=64, block=32, seqs=1, new=1, shortest=0, longest=0, back=0,
                none=0, ends=0, prompt=1, pad=0, scarce=False, lse=False, lens=0)


def _full(case):
    return {**DEFAULTS, **case}


def listed():
    return [
        # one decoding step of 64 requests: a row each, a page for every 16th of them
        dict(name="assign_step_64", op="assign", page=16, seqs=64, new=1, shortest=500, longest=4000),
        # a scheduler's turn over many requests, some of which have ended and are followed by prompts; a batch padded for replays
        dict(name="assign_turn_1000", op="assign", page=16, seqs=1000, new=1, shortest=1, longest=3000, ends=9, prompt=1500, pad=777),
        # one long prompt into an empty pool
        dict(name="assign_prompt", op="assign", page=64, seqs=1, ends=1, prompt=120000, shortest=1, longest=1),
        # a decoding step's rows appended to blocks that hold tokens already, and those blocks read: nothing but latency
        dict(name="store_step_fp8", op="store", form="fp8_blocks", seqs=64, new=1, shortest=500, longest=4000, back=32),
        # a prompt's rows as its prefill ends, written, and laid out again for an eviction pass
        dict(name="store_prompt_fp8", op="store", form="fp8_blocks", page=128, block=64, seqs=1, new=20000, shortest=20001,
             longest=20001, back=20000),
        # what an eviction pass kept of several prompts, 32 bits a value, to integer codes; no round length
        dict(name="store_budgets_int8", op="store", form="int8_blocks", dtype="fp32", h=16, hq=16, d=64, page=32, block=16, seqs=5,
             new=411, shortest=411, longest=911, back=411),
        # a step of 64 requests of uneven length: bound by the cache's read
        dict(name="attend_step_64_fp8", op="attend", form="fp8_blocks", seqs=64, new=1, shortest=400, longest=5000),
        # eight drafted tokens a request, seven query heads a key head, small pages
        dict(name="attend_drafts_int8", op="attend", form="int8_blocks", h=4, hq=28, page=16, block=16, seqs=16, new=8, shortest=1000,
             longest=9001, lse=True),
        # a chunk of a long prompt's prefill over what is already cached: the largest product
        dict(name="attend_chunk_fp8", op="attend", form="fp8_blocks", page=128, block=128, seqs=1, new=2000, shortest=24000, longest=24000),
        # one token of one request over an encoder's states: the smallest call
        dict(name="cross_step_1", op="cross", h=16, hq=16, d=64, seqs=1, new=1, shortest=1500, longest=1500),
        # a step of 64 requests, some of which have no states to look at, one query head a key head
        dict(name="cross_step_64", op="cross", h=16, hq=16, d=64, page=32, seqs=64, new=1, shortest=200, longest=1500, none=3, lse=True),
        # prompts of several requests over long states in 8 bits, a scale a block
        dict(name="cross_prompts_fp8", op="cross", form="fp8_blocks", h=8, hq=16, seqs=6, new=445, shortest=1000, longest=9000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above; odd sizes among them."""
    op = rng.choice(["assign", "store", "attend", "attend", "cross", "cross"])
    c = dict(op=op, lens=rng.randrange(1 << 30), page=rng.choice([16, 32, 64, 128]))
    if op == "assign":
        c.update(seqs=_log(rng, 1, 6000), new=rng.choice([1, 1, 1, rng.randint(2, 9)]), shortest=1, longest=_log(rng, 2, 4000))
        c.update(ends=rng.choice([0, 1, 2, 9, 50]), prompt=max(1, min(_log(rng, 1, 30000), 250000 // c["seqs"])))
        c.update(pad=rng.choice([0, 0, 1, _log(rng, 2, 2000)]), scarce=rng.random() < 0.3)
        return c
    c["h"], c["hq"] = rng.choice([(8, 32), (8, 32), (8, 16), (4, 28), (16, 16), (2, 8)])
    c["d"] = rng.choice([64, 80, 128, 128, 128])
    c["dtype"] = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    c["form"] = rng.choice(["fp8_blocks", "fp8_blocks", "int8_blocks"])
    c["block"] = rng.choice([b for b in (16, 32, 64, 128) if b <= c["page"]])
    if op == "store":
        c["seqs"] = rng.choice([1, 1, 4, 33])
        c["new"] = max(1, (_log(rng, 1, 16384) + rng.choice([0, 0, 1, 7])) // c["seqs"])
        c["shortest"] = c["new"]
        c["longest"] = c["new"] + rng.choice([0, 1, 500])
        c["back"] = max(1, min(c["new"], 4096))
        return c
    c["lse"] = rng.random() < 0.3
    if op == "cross":
        c["form"] = rng.choice(["plain", "plain", "fp8", "int8", "fp8_blocks", "int8_blocks"])
    kind = rng.choice(["one", "step", "step", "drafts", "chunk"])
    if kind == "one":
        c.update(seqs=1, new=1, longest=_log(rng, 1, 65536 if op == "attend" else 20000))
    elif kind == "chunk":
        c.update(seqs=rng.choice([1, 1, 2, 5]))
        c.update(new=_log(rng, 40, 1500 // c["seqs"]))
        c["longest"] = (c["new"] if op == "attend" else 0) + _log(rng, 1, 8000)
    else:
        c.update(seqs=_log(rng, 2, 64), new=rng.randint(2, 8) if kind == "drafts" else 1, longest=_log(rng, 100, 5000))
    c["shortest"] = max(c["new"] if op == "attend" else 1, c["longest"] // rng.choice([1, 2, 10]))
    c["longest"] = max(c["shortest"], c["longest"])
    if op == "cross" and c["seqs"] > 3:
        c["none"] = rng.choice([0, 1])
    return c


def _lengths(c):
    """(new rows, tokens) of every sequence.  Rows that look at another sequence's states are no tokens of it."""
    rng = random.Random(c["lens"])
    told = [rng.randint(c["shortest"], c["longest"]) for _ in range(c["seqs"])]
    return [(c["new"] or n, 0 if s < c["none"] else n) for s, n in enumerate(told)]


def _turn(c):
    """(tokens kept, tokens before, new rows) of every sequence of a scheduler's turn."""
    rng = random.Random(c["lens"])
    turn = []
    for s in range(c["seqs"]):
        n = rng.randint(c["shortest"], c["longest"])
        turn.append((0, n, rng.randint(max(1, c["prompt"] // 2), c["prompt"])) if c["ends"] and s % c["ends"] == c["ends"] - 1 else (n, n, c["new"]))
    return turn


def _pages(n, ps):
    return -(-n // ps)


def _type(c):
    return torch.float32 if c["dtype"] == "fp32" else torch.bfloat16


# ---- the operators in elementary operations ---------------------------------------------------------

def _assign(st):
    """Sequences ask in order.  One whose tokens would pass its table is refused, one whose rows the row tensors have no room for, and
    one that needs more pages than the ones before it have left; a refused sequence stays as it was and has no rows."""
    c, ps, table, stack = st["c"], st["c"]["page"], st["table"], st["free"]
    W, rows, pages = table.shape[1], st["rows"], stack.numel()
    had = st["before"].long().clamp(0, W * ps)
    want = torch.minimum(st["keep"].long().clamp(min=0), had) + st["new"].long()
    new = torch.where(want <= W * ps, st["new"].long(), 0)
    ok = (want <= W * ps) & ((new == 0) | (new.cumsum(0) <= rows))
    need = torch.where(ok, (want + ps - 1) // ps - (had + ps - 1) // ps, 0)
    take, give = need.clamp(min=0), (-need).clamp(min=0)
    taken, given = take.cumsum(0), give.cumsum(0)
    total = (st["n_free"].long() + given[-1]).clamp(max=pages)
    ok &= (take == 0) | (taken <= total)
    length = torch.where(ok, want, had)
    start = torch.nn.functional.pad(torch.where(ok, new, 0).cumsum(0), (1, 0))
    # pages that come back, and those that are dealt out, from the top of the stack down
    i = torch.arange(pages, device=DEV)
    s = torch.searchsorted(given, i, right=True).clamp(max=c["seqs"] - 1)
    page = st["table_and_one"][(s * W + (length[s] + ps - 1) // ps + i - (given - give)[s]).clamp(max=table.numel())]
    st["free_and_one"][torch.where(i < given[-1], total - 1 - i, pages)] = page
    out = torch.where(ok & (take > 0), taken, 0).amax()
    s = torch.searchsorted(taken, i, right=True).clamp(max=c["seqs"] - 1)
    at = s * W + (had[s] + ps - 1) // ps + i - (taken - take)[s]
    st["table_and_one"][torch.where(i < out, at, table.numel())] = stack[(total - 1 - i).clamp(min=0)]
    r = torch.arange(rows, device=DEV)
    s = torch.searchsorted(start[1:], r, right=True).clamp(max=c["seqs"] - 1)
    pos = (length[s] - start[s + 1] + r).clamp(0, W * ps - 1)
    none = r >= start[-1]
    slot = table[s, pos // ps].long() * ps + pos % ps
    return {"table": table, "free": stack, "n_free": (total - out).int().reshape(1), "seq_len": length.int(), "row_start": start.int(),
            "positions": torch.where(none, -1, pos).int(), "slots": torch.where(none, -1, slot).int()}


def _coded(form):
    return form.split("_")[0]


def _amax_scale(a, form):
    """The scale of values whose largest magnitude is a: for fp8 the least power of two that brings it to 448 or below, for
    int8 a / 127 rounded to 32 bits.  Zeros have none."""
    if form == "int8":
        return (a.double() / 127).float()
    m, e = torch.frexp(a)
    return torch.where(a > 0, torch.ldexp(torch.ones_like(a), e - torch.where(m <= 0.875, 9, 8)), 0.0)


def _codes(x, scale, form):
    """Codes of values x with these scales.  (In 64 bits: a quotient next to the middle of two codes must not be rounded twice.)"""
    y = x.double() / torch.where(scale > 0, scale, 1.0).double()
    return y.round().to(torch.int8) if form == "int8" else y.float().to(torch.float8_e4m3fn)


def _encode(x, form, block):
    """(codes, scales) of a pool's rows x [..., tokens, d]."""
    if form == "plain":
        return x, None
    kind, n = _coded(form), block if form.endswith("blocks") else 1
    y = x.float().reshape(*x.shape[:-2], x.shape[-2] // n, n * x.shape[-1])
    scale = _amax_scale(y.abs().amax(-1), kind)
    return _codes(y, scale[..., None], kind).reshape(x.shape), scale


def _bytes_of(t):
    return t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t


def _store(st, name):
    """Rows appended to blocks.  A block that begins with a new row takes its scale from its new rows alone; one that holds earlier
    tokens keeps its scale if it is enough, and otherwise their codes are rounded again, to the larger one."""
    c, kind, n, ps = st["c"], _coded(st["c"]["form"]), st["c"]["block"], st["c"]["page"]
    pool, scales = st[name + "pages"], st[name + "scale"]
    length, new = st["seq_len"].long(), st["start"][1:].long() - st["start"][:-1].long()
    first = length - new
    block = (first // n)[:, None] + torch.arange(st["most_blocks"], device=DEV)            # [seqs, blocks]
    pos = block[..., None] * n + torch.arange(n, device=DEV)                              # [seqs, blocks, tokens]
    fresh = (pos >= first[:, None, None]) & (pos < length[:, None, None])
    mine = block * n < length[:, None]
    row = (st["start"][:-1].long()[:, None, None] + pos - first[:, None, None]).clamp(0, st["rows"] - 1)
    page = torch.gather(st["table"].long(), 1, (block * n // ps).clamp(max=st["table"].shape[1] - 1))
    page = torch.where(mine, page, pool.shape[0] - 1)                                     # (the last page is nobody's)
    inside = pos % ps
    x = st[name][row].float().transpose(2, 3)                                             # [seqs, blocks, heads, tokens, d]
    a = torch.where(fresh[:, :, None, :, None], x.abs(), 0.0).amax((-1, -2))
    at = (block * n % ps) // n
    before = torch.where((block * n < first[:, None])[..., None], scales[page, :, at], 0.0)
    after = torch.maximum(before, _amax_scale(a, kind))
    old = _bytes_of(pool)[page[..., None], :, inside].view(pool.dtype).transpose(2, 3)   # [seqs, blocks, heads, tokens, d]
    again = _codes(old.double() * before.double()[..., None, None], after[..., None, None], kind)
    told = (pos < first[:, None, None])[:, :, None, :, None] & (after > before)[..., None, None]
    code = torch.where(told, _bytes_of(again), _bytes_of(old))
    code = torch.where(fresh[:, :, None, :, None], _bytes_of(_codes(x, after[..., None, None], kind)), code)
    _bytes_of(pool)[page[..., None], :, inside] = code.transpose(2, 3)
    scales[page, :, at] = after


def _read(st, name):
    """The last tokens of every sequence, [rows read, heads, d]."""
    c, ps = st["c"], st["c"]["page"]
    row = torch.arange(st["rows_back"], device=DEV)
    seq = torch.searchsorted(st["start_back"][1:], row, right=True)
    pos = st["seq_len"][seq] - st["start_back"][seq + 1] + row
    page, at = st["table"][seq, pos // ps].long(), pos % ps
    x = _bytes_of(st[name + "pages"])[page, :, at].view(st[name + "pages"].dtype).float()
    return (x * st[name + "scale"][page, :, at // c["block"]][..., None]).to(_type(c))


def _dense(st, name):
    """Keys or values of all sequences, [seqs, heads, longest, d] in 32 bits."""
    table = st["table"].long()
    x = _bytes_of(st[name + "pages"])[table].view(st[name + "pages"].dtype).float()
    S, n, h, ps, d = x.shape
    if st["c"]["form"] != "plain":
        scale = st[name + "scale"][table]
        x = (x.view(S, n, h, scale.shape[-1], -1, d) * scale[..., None, None]).view(x.shape)
    return x.transpose(1, 2).reshape(S, h, n * ps, d)


def _attend(st):
    c = st["c"]
    k, v = _dense(st, "K"), _dense(st, "V")
    S, h, L, d = k.shape
    G, most = c["hq"] // h, st["most_new"]
    start, new = st["start"][:-1].long(), st["start"][1:].long() - st["start"][:-1].long()
    t = torch.arange(most, device=DEV)
    q = st["Q"][(start[:, None] + t).clamp(max=st["rows"] - 1)].float()            # [S, most, hq, d]
    q = q.view(S, most, h, G, d).permute(0, 2, 3, 1, 4).reshape(S, h, G * most, d)
    x = (q @ k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(d)).view(S, h, G, most, L)
    sees = st["seq_len"].long()[:, None].expand(S, most)                            # how many positions each row sees
    if c["op"] == "attend":
        sees = sees - new[:, None] + t + 1
    seen = torch.arange(L, device=DEV) < sees[..., None]                            # [S, most, L]
    x.masked_fill_(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x = x.sub_(top.clamp(min=torch.finfo(torch.float32).min)).exp_()
    total = x.sum(-1, keepdim=True)
    o = (x.view(S, h, G * most, L) @ v).view(S, h, G, most, d) / torch.where(total > 0, total, 1.0)
    row = torch.arange(st["rows"], device=DEV)
    seq = torch.searchsorted(st["start"][1:], row, right=True)
    i = row - start[seq]
    out = {"out": o.permute(0, 3, 1, 2, 4).reshape(S, most, c["hq"], d)[seq, i].to(_type(c))}
    if c["lse"]:
        out["lse"] = (total.log() + top)[..., 0].permute(0, 3, 1, 2).reshape(S, most, c["hq"])[seq, i]
    return out


# ---- the same with the library's calls --------------------------------------------------------------

def _own(st):
    from paper_2509_00388_amd import binding as gk
    c = st["c"]
    if "params" not in st:      # what a serving loop keeps: the description of its batch, and scratch memory
        forms = {"plain": gk.PAGES_PLAIN, "fp8": gk.PAGES_FP8, "int8": gk.PAGES_INT8, "fp8_blocks": gk.PAGES_FP8_BLOCKS,
                 "int8_blocks": gk.PAGES_INT8_BLOCKS}
        p = dict(n_kv_heads=c["h"], n_q_heads=c["hq"], head_dim=c["d"], page_tokens=c["page"], n_seqs=c["seqs"],
                 table_pages=st["table"].shape[1], dtype=gk.FP32 if c["dtype"] == "fp32" else gk.BF16,
                 page_format=forms[c["form"]], scale_tokens=c["block"] if c["form"].endswith("blocks") else 0)
        n_pages = st["free"].numel() if c["op"] == "assign" else st["Kpages"].shape[0]
        p = st["params"] = gk.PagedParams(n_pages=n_pages, n_rows=st["rows"], max_rows=0 if c["op"] == "assign" else st["most_new"], **p)
        if c["op"] == "assign":
            st["ws"] = gk.alloc_assign_workspace(p, DEV)
        elif c["op"] == "store":
            st["params_back"] = gk.PagedParams(**{**p.__dict__, "n_rows": st["rows_back"], "max_rows": st["most_back"]})
        else:
            st["ws"] = gk.alloc_attend_workspace(p, DEV)
    p = st["params"]
    if c["op"] == "assign":
        gk.graphkv_cache_assign(p, st["new"], st["before"], st["table"], st["free"], st["n_free"], keep=st["keep"], seq_len=st["seq_len"],
                                free_after=st["free_after"], row_start=st["start"], positions=st["positions"], slots=st["slots"], ws=st["ws"])
        return {"table": st["table"], "free": st["free"], "n_free": st["free_after"], "seq_len": st["seq_len"], "row_start": st["start"],
                "positions": st["positions"], "slots": st["slots"]}
    pools = (st["Kpages"], st["Vpages"], st["table"], st["seq_len"])
    scales = (st.get("Kscale"), st.get("Vscale"))
    if c["op"] == "store":
        gk.graphkv_cache_write(p, st["K"], st["V"], *pools, st["start"], *scales)
        k, v = gk.graphkv_cache_read(st["params_back"], *pools, st["start_back"], *scales)
        return {"K": k, "V": v}
    lse = torch.empty(st["rows"], c["hq"], dtype=torch.float32, device=DEV) if c["lse"] else None
    call = gk.graphkv_attend if c["op"] == "attend" else gk.graphkv_cross_attend
    out = call(p, st["Q"], *pools, st["start"], *scales, lse=lse, ws=st["ws"])
    return {"out": out, "lse": lse} if c["lse"] else {"out": out}


# ---- cases ------------------------------------------------------------------------------------------

def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _starts(counts):
    return list(itertools.accumulate(counts, initial=0))


def _prepare_assign(c, g):
    turn = _turn(c)
    ps = c["page"]
    width = max(_pages(max(had, keep + new), ps) for keep, had, new in turn)
    held = sum(_pages(had, ps) for _, had, _ in turn)
    asked = sum(max(0, _pages(keep + new, ps) - _pages(had, ps)) for keep, had, new in turn)
    back = sum(max(0, _pages(had, ps) - _pages(keep + new, ps)) for keep, had, new in turn)
    spare = max(0, asked - back)
    spare = spare // 2 if c["scarce"] else spare + spare // 3 + 5
    pages = held + spare
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    # (both have one entry more, which the plain form writes to in place of nothing)
    table = torch.zeros(c["seqs"] * width + 1, dtype=torch.int32, device=DEV)
    n_held = torch.tensor([_pages(had, ps) for _, had, _ in turn], device=DEV)
    held_by = torch.repeat_interleave(torch.arange(c["seqs"], device=DEV), n_held)
    table[held_by * width + torch.arange(held, device=DEV) - (n_held.cumsum(0) - n_held)[held_by]] = order[:held]
    stack = torch.zeros(pages + 1, dtype=torch.int32, device=DEV)
    stack[:spare] = order[held:]
    rows = sum(new for _, _, new in turn) + c["pad"]
    empty = lambda n: torch.empty(n, dtype=torch.int32, device=DEV)  # noqa: E731
    return dict(c=c, rows=rows, table_and_one=table, table=table[:-1].view(c["seqs"], width), free_and_one=stack, free=stack[:-1],
                n_free=_ints([spare]), keep=_ints([k for k, _, _ in turn]), before=_ints([n for _, n, _ in turn]),
                new=_ints([n for _, _, n in turn]), seq_len=empty(c["seqs"]), start=empty(c["seqs"] + 1), free_after=empty(1),
                positions=empty(rows), slots=empty(rows))


def _rows(c, n, g):
    """K, V and Q rows, as slices of one projection's output; some channels of K are much larger, as they are behind rotary
    positions, and tokens differ in size."""
    h, hq, d = c["h"], c["hq"], c["d"]
    x = torch.randn(n, hq + 2 * h, d, generator=g, device=DEV)
    x[:, hq:] *= torch.exp(0.5 * torch.randn(n, 1, 1, generator=g, device=DEV))
    x = x.to(_type(c))
    q, k, v = x[:, :hq], x[:, hq:hq + h], x[:, hq + h:]
    k[..., 1::d // 4] *= 8.0
    q[..., 1::d // 4] *= 0.25
    return k, v, q


def prepare(case, seed):
    c = _full(case)
    g = torch.Generator(device=DEV).manual_seed(seed)
    if c["op"] == "assign":
        return _prepare_assign(c, g)
    pairs = _lengths(c)
    ps, h, d = c["page"], c["h"], c["d"]
    need = [_pages(n, ps) for _, n in pairs]
    pages, width = sum(need) + 3, max(need + [1])
    order = (torch.randperm(pages - 1, generator=g, device=DEV)[:sum(need)]).to(torch.int32)   # (the last page is nobody's)
    table = torch.zeros(len(pairs), width, dtype=torch.int32, device=DEV)
    first = 0
    for s, n in enumerate(need):
        table[s, :n] = order[first:first + n]
        first += n
    starts = _starts([new for new, _ in pairs])
    st = dict(c=c, rows=starts[-1], most_new=max(new for new, _ in pairs), table=table, seq_len=_ints([n for _, n in pairs]),
              start=_ints(starts))
    # what the pool holds: rows of the same kind, encoded
    for i, name in enumerate("KV"):
        x = _rows({**c, "hq": 0}, pages * ps, g)[i].reshape(pages, ps, h, d).transpose(1, 2).contiguous()
        code, scale = _encode(x, c["form"], c["block"])
        st[name + "pages"] = code.contiguous()
        if scale is not None:
            st[name + "scale"] = scale.contiguous()
    k, v, q = _rows(c, st["rows"], g)
    if c["op"] == "store":
        back = [min(n, c["back"]) for _, n in pairs]
        n = c["block"]
        st.update(K=k, V=v, start_back=_ints(_starts(back)), rows_back=sum(back), most_back=max(back),
                  most_blocks=max((length - 1) // n - (length - new) // n + 1 for new, length in pairs))
    else:
        st["Q"] = q
    return st


def run(st):
    if own:
        return _own(st)
    if st["c"]["op"] == "assign":
        return _assign(st)
    if st["c"]["op"] == "store":
        _store(st, "K")
        _store(st, "V")
        return {"K": _read(st, "K"), "V": _read(st, "V")}
    return _attend(st)


def work(case):
    c = _full(case)
    if c["op"] == "assign":
        turn, ps = _turn(c), c["page"]
        moved = sum(abs(_pages(keep + new, ps) - _pages(had, ps)) for keep, had, new in turn)
        rows = sum(new for _, _, new in turn) + c["pad"]
        # lengths, what is kept and asked for; lengths and row numbers; a page number from one place to another; two numbers a row
        return {"bytes": 20 * c["seqs"] + 8 * moved + 8 * rows + 16, "flops": 0}
    pairs = _lengths(c)
    h, hq, d = c["h"], c["hq"], c["d"]
    e = 4 if c["dtype"] == "fp32" else 2
    each = {"plain": d * e, "fp8": d + 4, "int8": d + 4}.get(c["form"], d + 4 / c["block"])      # bytes of a cached row
    rows = sum(new for new, _ in pairs)
    if c["op"] == "store":
        back = sum(min(n, c["back"]) for _, n in pairs)
        return {"bytes": 2 * h * (rows + back) * (d * e + each), "flops": 0}
    nbytes = sum(n for _, n in pairs) * h * 2 * each + 2 * rows * hq * d * e + (4 * rows * hq if c["lse"] else 0)
    seen = sum(new * n - (new * (new - 1) // 2 if c["op"] == "attend" else 0) for new, n in pairs)
    return {"bytes": nbytes, "flops": 4 * hq * d * seen}


# ---- the definitions in 64 bits ---------------------------------------------------------------------

def _exact_codes(x, s, kind):
    """The values, before the scale, of the codes of x in 64 bits."""
    y = x / torch.where(s > 0, s, 1.0)
    if kind == "int8":
        return torch.round(y)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)      # e4m3: 3 bits behind the first
    return torch.round(y / step) * step


def _exact_scale(a, kind):
    return (a / 127).float().double() if kind == "int8" else torch.exp2(torch.ceil(torch.log2(a / 448)))


def exact(case, seed):
    st = prepare(case, seed)
    c = st["c"]
    ps, h, d, n_block = c["page"], c["h"], c["d"], c["block"]

    def assign():
        """One sequence after the other."""
        rows = st["rows"]
        table, stack = st["table"].cpu(), st["free"].cpu()
        free = stack[:int(st["n_free"])].tolist()
        W = table.shape[1]
        turn = list(zip(st["keep"].tolist(), st["before"].tolist(), st["new"].tolist()))
        asked, ok = 0, []
        for keep, had, new in turn:
            fits = keep + new <= W * ps
            asked += new if fits else 0
            ok.append(fits and (new == 0 or asked <= rows))
        short = 0
        back = []      # pages that come back, in the order in which they would be taken again
        for s, (keep, had, new) in enumerate(turn):
            if ok[s]:
                back += table[s, _pages(keep + new, ps):_pages(had, ps)].tolist()
        free += back[::-1]
        stack[:len(free)] = torch.tensor(free, dtype=torch.int32)
        for s, (keep, had, new) in enumerate(turn):
            need = _pages(keep + new, ps) - _pages(had, ps) if ok[s] else 0
            if need > 0 and (short or need > len(free)):
                ok[s], short = False, 1
            elif need > 0:
                for i in range(need):
                    table[s, _pages(had, ps) + i] = free.pop()
        length = [keep + new if ok[s] else had for s, (keep, had, new) in enumerate(turn)]
        start = _starts([new if ok[s] else 0 for s, (_, _, new) in enumerate(turn)])
        pos, slot = torch.full((rows,), -1), torch.full((rows,), -1)
        for s in range(len(turn)):
            t = torch.arange(length[s] - (start[s + 1] - start[s]), length[s])
            pos[start[s]:start[s + 1]] = t
            slot[start[s]:start[s + 1]] = table[s].long()[t // ps] * ps + t % ps
        return {"table": table, "free": stack, "n_free": torch.tensor([len(free)]), "seq_len": torch.tensor(length), "row_start": torch.tensor(start),
                "positions": pos, "slots": slot}

    if c["op"] == "assign":
        return assign()
    pairs = _lengths(c)

    def rows_of(name, s, first, last):
        """Values of positions first .. last - 1 in 64 bits, [tokens, heads, d]."""
        t = torch.arange(first, last, device=DEV)
        page = st["table"][s].long()[t // ps]
        x = _bytes_of(st[name + "pages"])[page, :, t % ps].view(st[name + "pages"].dtype).double()
        if c["form"] == "plain":
            return x
        scale = st[name + "scale"].double()
        return x * scale[page, :, (t % ps) // (ps // scale.shape[-1])][..., None]

    if c["op"] == "store":
        kind, back = _coded(c["form"]), {}
        for name in "KV":
            got, row = [], 0
            for s, (new, length) in enumerate(pairs):
                x = st[name][row:row + new].double()
                row += new
                first = length - new
                begin = first // n_block * n_block
                if begin < first:      # a block that holds earlier tokens
                    page, at = int(st["table"][s, begin // ps]), begin % ps
                    before = st[name + "scale"][page, :, at // n_block].double()
                    inside = x[:n_block - (first - begin)]
                    after = torch.maximum(before, _exact_scale(inside.abs().amax((0, 2)), kind))[None, :, None]
                    old = _exact_codes(rows_of(name, s, begin, first), after, kind) * after
                    x = torch.cat([old, _exact_codes(inside, after, kind) * after, x[inside.shape[0]:]])
                    done = old.shape[0] + inside.shape[0]
                else:
                    done = 0
                rest = x[done:]
                full = rest.shape[0] // n_block * n_block
                parts = [x[:done]]
                for y in (rest[:full].reshape(-1, n_block, h, d), rest[full:][None]):
                    if y.numel():
                        scale = _exact_scale(y.abs().amax((1, 3)), kind)[:, None, :, None]
                        parts.append((_exact_codes(y, scale, kind) * scale).reshape(-1, h, d))
                x = torch.cat(parts)
                want = min(length, c["back"])
                have = x.shape[0]
                got.append(x[have - want:] if want <= have else torch.cat([rows_of(name, s, length - want, length - have), x]))
            back[name] = torch.cat(got)
        return back
    G = c["hq"] // h
    out = torch.zeros(st["rows"], c["hq"], d, dtype=torch.float64, device=DEV)
    lse = torch.full((st["rows"], c["hq"]), -math.inf, dtype=torch.float64, device=DEV)
    first = 0
    for s, (new, n) in enumerate(pairs):
        if n:
            k, v = rows_of("K", s, 0, n), rows_of("V", s, 0, n)
            last = torch.arange(n - new, n, device=DEV) if c["op"] == "attend" else torch.full((new,), n - 1, device=DEV)
            hidden = torch.arange(n, device=DEV)[None, :] > last[:, None]
            for q in range(c["hq"]):
                x = st["Q"][first:first + new, q].double() @ k[:, q // G].T.contiguous() / math.sqrt(d)
                x = x.masked_fill(hidden, -math.inf)
                lse[first:first + new, q] = torch.logsumexp(x, -1)
                out[first:first + new, q] = torch.softmax(x, -1) @ v[:, q // G].contiguous()
        first += new
    return {"out": out, "lse": lse} if c["lse"] else {"out": out}
