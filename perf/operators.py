"""The paged cache's operators as they are timed and checked: writing rows to pages, reading them back, attention.

A batch is told the same way to each of them.  `table` [seqs, pages of the longest] names the pages of a sequence in a pool
[pages, key-value heads, tokens a page, d]; `seq_len` holds how many tokens a sequence has, its new ones included; rows
start[s] to start[s + 1] - 1 of the row tensors [rows, heads, d] are the last tokens of sequence s.

`run()` computes a case with elementary torch operations, or, where `own` is set, with the library's calls.  `listed()` holds
the fixed cases, `draw()` gives further ones of the same ranges, `exact()` the results in 64 bits.

Fields of a case: op (write: rows to pages, returned as the pools; store: written and read back; read; attend), form of the
pages (plain: the rows' type; fp8; int8), dtype of the rows, h / hq key-value and query heads, d head dimension, page tokens a
page, seqs sequences of `new` new rows each, with shortest to longest tokens, the last of them with chunk new rows of
chunk_len tokens where these are given; by_head: rows lie head after head, as the eviction pass leaves them, and not as
slices of one projection's output; lse: the logarithm of the softmax sums is returned too; lens: draws the lengths.
"""
import math
import random

import torch

own = False

DEV = "cuda"
DEFAULTS = dict(form="plain", dtype="bf16", h=8, hq=32, d=128, page=64, seqs=1, new=1, shortest=0, longest=0, chunk=0,
                chunk_len=0, by_head=False, lse=False, lens=0)


def _full(case):
    return {**DEFAULTS, **case}


def listed():
    return [
        # one decoding step's rows of 64 requests: nothing but latency
        dict(name="write_step_fp8", op="write", form="fp8", seqs=64, new=1, shortest=500, longest=4000),
        # a prompt's rows as its prefill ends, straight from the projection's output
        dict(name="write_prompt_fp8", op="write", form="fp8", seqs=1, new=32768, shortest=32768, longest=32768),
        # what the eviction pass kept of a prompt, 32 bits a value, written to 8-bit pages and read back; odd budget
        dict(name="store_budget_int8", op="store", form="int8", dtype="fp32", h=16, hq=16, d=64, page=32, seqs=1, new=2011,
             shortest=2011, longest=2011, by_head=True),
        # a paged prompt laid out head after head, as the eviction pass takes it
        dict(name="read_32k_fp8", op="read", form="fp8", seqs=1, new=32768, shortest=32768, longest=32768, by_head=True),
        # several short prompts of no round length, plain pages
        dict(name="read_ragged", op="read", h=4, hq=28, page=16, seqs=9, new=0, shortest=100, longest=3000),
        # one request's step over an evicted cache: the smallest call
        dict(name="attend_step_2k", op="attend", seqs=1, new=1, shortest=2048, longest=2048),
        # a step of 64 requests of uneven length over 8-bit pages
        dict(name="attend_step_64_fp8", op="attend", form="fp8", seqs=64, new=1, shortest=400, longest=5000),
        # one request's step over a long context that nothing was evicted from
        dict(name="attend_step_128k", op="attend", seqs=1, new=1, shortest=131072, longest=131072),
        # eight drafted tokens a request, seven query heads a key head, 8-bit integers
        dict(name="attend_drafts_int8", op="attend", form="int8", h=4, hq=28, page=16, seqs=16, new=8, shortest=1000,
             longest=9001, lse=True),
        # a chunk of a long prompt's prefill over what is already cached: the largest product
        dict(name="attend_chunk_32k", op="attend", seqs=1, new=2048, shortest=32768, longest=32768),
        # a chunk of one prompt beside the steps of others, one query head a key head
        dict(name="attend_mixed_fp8", op="attend", form="fp8", h=16, hq=16, page=32, seqs=13, new=1, shortest=300,
             longest=4500, chunk=500, chunk_len=5003),
        # 32 bits throughout, heads of 64, a chunk of no round length
        dict(name="attend_chunk_fp32_d64", op="attend", dtype="fp32", h=16, hq=16, d=64, seqs=2, new=701, shortest=2000,
             longest=5001, lse=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above; odd sizes among them."""
    op = rng.choice(["write", "store", "read", "attend", "attend", "attend", "attend", "attend"])
    h, hq = rng.choice([(8, 32), (8, 32), (8, 16), (4, 28), (16, 16), (2, 8)])
    c = dict(op=op, h=h, hq=hq, d=rng.choice([64, 80, 128, 128, 128]), page=rng.choice([16, 32, 64, 128]),
             lens=rng.randrange(1 << 30))
    c["form"] = rng.choice(["plain", "plain", "fp8", "fp8", "int8"] if op != "store" else ["fp8", "int8"])
    c["dtype"] = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    if op == "write" and c["form"] == "int8":
        c["form"] = "plain"
    if op != "attend":
        c["by_head"] = rng.random() < 0.5
        c["seqs"] = rng.choice([1, 1, 4, 33])
        total = _log(rng, 1, 16384) + rng.choice([0, 0, 1, 7])
        if op == "read":
            c["longest"] = max(1, total // c["seqs"])
            c["shortest"] = max(1, c["longest"] // 4)
            c["new"] = 0
        else:
            c["new"] = max(1, total // c["seqs"])
            c["longest"] = c["new"] + rng.choice([0, 1, 500])
            c["shortest"] = c["new"]
        return c
    c["lse"] = rng.random() < 0.3
    kind = rng.choice(["one", "step", "step", "drafts", "chunk", "mixed"])
    if kind == "one":
        c.update(seqs=1, new=1, longest=_log(rng, 1, 131072))
    elif kind == "chunk":
        c.update(seqs=rng.choice([1, 1, 2]), new=_log(rng, 40, 1500))
        c["longest"] = c["new"] + _log(rng, 1, 8000)
    else:
        c.update(seqs=_log(rng, 2, 64), new=rng.randint(2, 8) if kind == "drafts" else 1, longest=_log(rng, 100, 5000))
        if kind == "mixed":
            c.update(seqs=rng.randint(2, 12), chunk=_log(rng, 40, 500))
            c["chunk_len"] = c["chunk"] + _log(rng, 1, 4500)
    c["shortest"] = max(c["new"], c["longest"] // rng.choice([1, 2, 10]))
    c["longest"] = max(c["shortest"], c["longest"])
    return c


def _lengths(c):
    """(new rows, tokens) of every sequence; a read takes all of a sequence's rows."""
    rng = random.Random(c["lens"])
    told = [rng.randint(c["shortest"], c["longest"]) for _ in range(c["seqs"])]
    pairs = [(c["new"] or n, n) for n in told]
    if c["chunk"]:
        pairs[-1] = (c["chunk"], c["chunk_len"])
    return pairs


def _type(c):
    return torch.float32 if c["dtype"] == "fp32" else torch.bfloat16


# ---- the operators in elementary operations ---------------------------------------------------------

def _amax_scale(a, form):
    """The scale of rows whose largest magnitude is a: for fp8 the least power of two that brings it to 448 or below, for
    int8 a / 127 rounded to 32 bits.  Rows of zeros have none."""
    if form == "int8":
        return (a.double() / 127).float()
    m, e = torch.frexp(a)
    return torch.where(a > 0, torch.ldexp(torch.ones_like(a), e - torch.where(m <= 0.875, 9, 8)), 0.0)


def _encode(x, form):
    """(codes, scales) of rows x [..., d]."""
    if form == "plain":
        return x, None
    x = x.float()
    scale = _amax_scale(x.abs().amax(-1), form)
    # (in 64 bits: a quotient next to the middle of two integers must not be rounded twice)
    y = x.double() / torch.where(scale > 0, scale, 1.0).double()[..., None]
    return (y.round().to(torch.int8) if form == "int8" else y.float().to(torch.float8_e4m3fn)), scale


def _places(st):
    """Page, place within it and sequence of every row."""
    row = torch.arange(st["rows"], device=DEV)
    seq = torch.searchsorted(st["start"][1:], row, right=True)
    at = st["seq_len"][seq] - st["start"][seq + 1] + row
    return st["table"][seq, at // st["c"]["page"]].long(), at % st["c"]["page"], seq


def _bytes_of(t):
    return t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t


def _write(st, name):
    page, at, _ = _places(st)
    code, scale = _encode(st[name], st["c"]["form"])
    _bytes_of(st[name + "pages"])[page, :, at] = _bytes_of(code)
    if scale is not None:
        st[name + "scale"][page, :, at] = scale


def _read(st, name):
    page, at, _ = _places(st)
    x = _bytes_of(st[name + "pages"])[page, :, at].view(st[name + "pages"].dtype).float()
    if st["c"]["form"] != "plain":
        x = x * st[name + "scale"][page, :, at][..., None]
    x = x.to(_type(st["c"]))
    return x.transpose(0, 1).contiguous().transpose(0, 1) if st["c"]["by_head"] else x


def _dense(st, name):
    """Keys or values of all sequences, [seqs, heads, longest, d] in 32 bits."""
    x = _bytes_of(st[name + "pages"])[st["table"].long()].view(st[name + "pages"].dtype).float()
    if st["c"]["form"] != "plain":
        x = x * st[name + "scale"][st["table"].long()][..., None]
    S, n, h, ps, d = x.shape
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
    x = (q @ k.transpose(2, 3)).mul_(1.0 / math.sqrt(d)).view(S, h, G, most, L)
    last = (st["seq_len"].long() - new)[:, None] + t                                # position of each row
    seen = torch.arange(L, device=DEV) <= last[..., None]                           # [S, most, L]
    x.masked_fill_(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    o = (x.view(S, h, G * most, L) @ v).view(S, h, G, most, d) / total
    seq = _places(st)[2]
    i = torch.arange(st["rows"], device=DEV) - start[seq]
    out = {"out": o.permute(0, 3, 1, 2, 4).reshape(S, most, c["hq"], d)[seq, i].to(_type(c))}
    if c["lse"]:
        out["lse"] = (total.log() + top)[..., 0].permute(0, 3, 1, 2).reshape(S, most, c["hq"])[seq, i]
    return out


# ---- the same with the library's calls --------------------------------------------------------------

def _own(st):
    from paper_2509_00388_amd import binding as gk
    c = st["c"]
    if "params" not in st:      # what a serving loop keeps: the description of its batch, and scratch memory
        p = st["params"] = gk.PagedParams(
            n_kv_heads=c["h"], n_q_heads=c["hq"], head_dim=c["d"], page_tokens=c["page"], n_pages=st["Kpages"].shape[0],
            n_seqs=st["table"].shape[0], table_pages=st["table"].shape[1], n_rows=st["rows"], max_rows=st["most_new"],
            dtype=gk.FP32 if c["dtype"] == "fp32" else gk.BF16,
            page_format={"plain": gk.PAGES_PLAIN, "fp8": gk.PAGES_FP8, "int8": gk.PAGES_INT8}[c["form"]])
        if c["op"] == "attend":
            st["ws"] = gk.alloc_attend_workspace(p, DEV)
    p = st["params"]
    batch = (st["table"], st["seq_len"], st["start"])
    pools = (st["Kpages"], st["Vpages"])
    scales = (st.get("Kscale"), st.get("Vscale"))
    if c["op"] == "attend":
        lse = torch.empty(st["rows"], c["hq"], dtype=torch.float32, device=DEV) if c["lse"] else None
        out = gk.graphkv_attend(p, st["Q"], *pools, *batch, *scales, lse=lse, ws=st["ws"])
        return {"out": out, "lse": lse} if c["lse"] else {"out": out}
    if c["op"] in ("write", "store"):
        gk.graphkv_cache_write(p, st["K"], st["V"], *pools, *batch, *scales)
    if c["op"] in ("read", "store"):
        into = [None, None]
        if c["by_head"]:
            into = [torch.empty(c["h"], st["rows"], c["d"], dtype=_type(c), device=DEV).transpose(0, 1) for _ in range(2)]
        k, v = gk.graphkv_cache_read(p, *pools, *batch, *scales, *into)
        return {"K": k, "V": v}
    return None


# ---- cases ------------------------------------------------------------------------------------------

def _rows(c, n, g, scale=1.0):
    """K, V and Q rows, as slices of one projection's output or head after head; some channels of K are much larger, as
    they are behind rotary positions."""
    h, hq, d = c["h"], c["hq"], c["d"]
    if c["by_head"]:
        k, v, q = (torch.randn(m, n, d, generator=g, device=DEV).to(_type(c)).transpose(0, 1) for m in (h, h, hq))
    else:
        x = torch.randn(n, hq + 2 * h, d, generator=g, device=DEV).to(_type(c))
        q, k, v = x[:, :hq], x[:, hq:hq + h], x[:, hq + h:]
    k[..., 1::d // 4] *= 8.0
    q[..., 1::d // 4] *= 0.25
    return k, v, q


def prepare(case, seed):
    c = _full(case)
    g = torch.Generator(device=DEV).manual_seed(seed)
    pairs = _lengths(c)
    ps, h, d = c["page"], c["h"], c["d"]
    need = [-(-n // ps) for _, n in pairs]
    pages, width = sum(need) + 3, max(need)
    order = torch.randperm(pages, generator=g, device=DEV)[:sum(need)].to(torch.int32)
    table = torch.zeros(len(pairs), width, dtype=torch.int32, device=DEV)
    first = 0
    for s, n in enumerate(need):
        table[s, :n] = order[first:first + n]
        first += n
    starts = [0]
    for new, _ in pairs:
        starts.append(starts[-1] + new)
    st = dict(c=c, rows=starts[-1], most_new=max(new for new, _ in pairs), table=table,
              seq_len=torch.tensor([n for _, n in pairs], dtype=torch.int32, device=DEV),
              start=torch.tensor(starts, dtype=torch.int32, device=DEV))
    # what the pool holds: rows of the same kind, encoded
    for i, name in enumerate("KV"):
        x = _rows({**c, "by_head": False}, pages * ps, g)[i].reshape(pages, ps, h, d).transpose(1, 2).contiguous()
        code, scale = _encode(x, c["form"])
        st[name + "pages"] = code.contiguous()
        if scale is not None:
            st[name + "scale"] = scale.contiguous()
    if c["op"] != "read":
        k, v, q = _rows(c, st["rows"], g)
        st.update({"Q": q} if c["op"] == "attend" else {"K": k, "V": v})
    return st


def _pools(st):
    names = ("Kpages", "Vpages") if st["c"]["form"] == "plain" else ("Kpages", "Vpages", "Kscale", "Vscale")
    return {n: st[n] for n in names}


def run(st):
    op = st["c"]["op"]
    if own:
        out = _own(st)
        return _pools(st) if op == "write" else out
    if op == "attend":
        return _attend(st)
    if op in ("write", "store"):
        _write(st, "K")
        _write(st, "V")
    return _pools(st) if op == "write" else {"K": _read(st, "K"), "V": _read(st, "V")}


def work(case):
    c = _full(case)
    pairs = _lengths(c)
    h, hq, d = c["h"], c["hq"], c["d"]
    e = 4 if c["dtype"] == "fp32" else 2
    cached = d * e if c["form"] == "plain" else d + 4                # bytes of a cached row
    rows = sum(new for new, _ in pairs)
    if c["op"] != "attend":
        moved = 2 * rows * h * (d * e + cached)
        return {"bytes": moved * (2 if c["op"] == "store" else 1), "flops": 0}
    nbytes = sum(n for _, n in pairs) * h * 2 * cached + 2 * rows * hq * d * e + (4 * rows * hq if c["lse"] else 0)
    seen = sum(new * (n - new) + new * (new + 1) // 2 for new, n in pairs)
    return {"bytes": nbytes, "flops": 4 * hq * d * seen}


# ---- the definitions in 64 bits ---------------------------------------------------------------------

def _exact_codes(x, form):
    """Values that 8-bit codes stand for before the scale, and the scales, of rows x in 64 bits."""
    a = x.abs().amax(-1)
    if form == "int8":
        s = a / 127
        return torch.round(x / s.float().double()[..., None]), s
    s = torch.exp2(torch.ceil(torch.log2(a / 448)))
    y = x / s[..., None]
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)      # e4m3: 3 bits behind the first
    return torch.round(y / step) * step, s


def exact(case, seed):
    st = prepare(case, seed)
    c = st["c"]
    pairs = _lengths(c)
    ps, h, d, form = c["page"], c["h"], c["d"], c["form"]
    pool = {n: st[n].double() for n in _pools(st)}
    where = [st["table"][s].long()[torch.arange(n - new if c["op"] != "attend" else 0, n, device=DEV) // ps]
             for s, (new, n) in enumerate(pairs)]
    inside = [torch.arange(n - new if c["op"] != "attend" else 0, n, device=DEV) % ps for new, n in pairs]

    def rows_of(name, s):
        x = pool[name + "pages"][where[s], :, inside[s]]
        return x if form == "plain" else x * pool[name + "scale"][where[s], :, inside[s]][..., None]

    if c["op"] == "read":
        return {n: torch.cat([rows_of(n, s) for s in range(len(pairs))]) for n in "KV"}
    if c["op"] in ("write", "store"):
        page, at = torch.cat(where), torch.cat(inside)
        back = {}
        for n in "KV":
            x = st[n].double()
            code, scale = (x, None) if form == "plain" else _exact_codes(x, form)
            pool[n + "pages"][page, :, at] = code
            if scale is not None:
                pool[n + "scale"][page, :, at] = scale
            back[n] = x if scale is None else code * scale[..., None]
        return pool if c["op"] == "write" else back
    G = c["hq"] // h
    out = torch.empty(st["rows"], c["hq"], d, dtype=torch.float64, device=DEV)
    lse = torch.empty(st["rows"], c["hq"], dtype=torch.float64, device=DEV)
    first = 0
    for s, (new, n) in enumerate(pairs):
        k, v = rows_of("K", s), rows_of("V", s)
        hidden = torch.arange(n, device=DEV)[None, :] > torch.arange(n - new, n, device=DEV)[:, None]
        for q in range(c["hq"]):
            x = st["Q"][first:first + new, q].double() @ k[:, q // G].T.contiguous() / math.sqrt(d)
            x = x.masked_fill(hidden, -math.inf)
            lse[first:first + new, q] = torch.logsumexp(x, -1)
            out[first:first + new, q] = torch.softmax(x, -1) @ v[:, q // G].contiguous()
        first += new
    return {"out": out, "lse": lse} if c["lse"] else {"out": out}
