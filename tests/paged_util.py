"""Batches of sequences in a paged cache for tests, and the operators' definitions in 64 bits on the CPU."""
import math

import torch

from paper_2509_00388_amd import binding as gk

TORCH = {gk.FP32: torch.float32, gk.BF16: torch.bfloat16}
CODE = {gk.PAGES_FP8: torch.float8_e4m3fn, gk.PAGES_INT8: torch.int8}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def encode(x, form):
    """Codes (as the values they stand for before the scale) and 32-bit scales of rows x, from the definition."""
    x = x.double()
    a = x.abs().amax(-1)
    none = a < 2.0 ** -100
    if form == gk.PAGES_INT8:
        s = (a / 127).float().double()
        s[none] = 0.0
        y = torch.where(none[..., None], 0.0, x / torch.where(none, 1.0, s)[..., None])
        return y.round(), s
    k = torch.ceil(torch.log2(torch.where(none, 1.0, a) / 448))
    k = torch.where(448 * torch.exp2(k - 1) >= a, k - 1, torch.where(448 * torch.exp2(k) < a, k + 1, k))   # (log2 is rounded)
    s = torch.where(none, 0.0, torch.exp2(k))
    y = torch.where(none[..., None], 0.0, x / torch.where(none, 1.0, s)[..., None])
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(y / step) * step, s


class Batch:
    """Sequences of (new rows, tokens); row tensors begin with `before` rows of no sequence and end with `behind`."""

    def __init__(self, pairs, H=2, G=1, d=64, ps=16, dtype=gk.BF16, form=gk.PAGES_PLAIN, before=0, behind=0, seed=0, impl=0,
                 max_rows=None, spare=2, table_pages=None):
        self.pairs, self.H, self.G, self.d, self.ps, self.dtype, self.form = pairs, H, G, d, ps, dtype, form
        self.g = torch.Generator().manual_seed(seed)
        need = [-(-n // ps) for _, n in pairs]
        pages = sum(need) + spare
        width = table_pages or max(need + [1])
        order = torch.randperm(pages, generator=self.g)
        self.table = torch.randint(0, pages, (len(pairs), width), generator=self.g).int()   # (unused entries name some page)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = order[at:at + n].int()
            at += n
        starts = [before]
        for n, _ in pairs:
            starts.append(starts[-1] + n)
        self.rows = starts[-1] + behind
        self.start = torch.tensor(starts, dtype=torch.int32)
        self.len = torch.tensor([n for _, n in pairs], dtype=torch.int32)
        self.p = gk.PagedParams(n_kv_heads=H, n_q_heads=H * G, head_dim=d, page_tokens=ps, n_pages=pages, n_seqs=len(pairs),
                                table_pages=width, n_rows=self.rows, max_rows=max_rows or max([n for n, _ in pairs] + [0]),
                                dtype=dtype, page_format=form, impl=impl)
        self.pool = {}
        for n in "KV":
            x = torch.randn(pages, H, ps, d, generator=self.g).to(TORCH[dtype])
            if n == "K":
                x[..., 3::d // 2] *= 5
            self.set_pool(n, x)

    def set_pool(self, n, x):
        if self.form == gk.PAGES_PLAIN:
            self.pool[n] = x
        else:
            code, s = encode(x.double(), self.form)
            self.pool[n] = code.to(torch.int8) if self.form == gk.PAGES_INT8 else code.float().to(torch.float8_e4m3fn)
            self.pool[n + "s"] = s.float()

    def random_rows(self, heads, by_head=False, fused=0):
        """Rows [rows, heads, d]: packed, head after head, or a slice of wider rows."""
        if by_head:
            return torch.randn(heads, self.rows, self.d, generator=self.g).to(TORCH[self.dtype]).transpose(0, 1)
        wide = torch.randn(self.rows, heads + fused, self.d, generator=self.g).to(TORCH[self.dtype])
        return wide[:, fused:] if fused else wide

    def values(self, n):
        """The pool's values in 64 bits."""
        x = self.pool[n].double()
        return x if self.form == gk.PAGES_PLAIN else x * self.pool[n + "s"].double()[..., None]

    def place(self, s, pos):
        """(page, place in it) of a position, None if it has none."""
        if pos < 0 or pos >= self.table.shape[1] * self.ps:
            return None
        page = int(self.table[s, pos // self.ps])
        return (page, pos % self.ps) if 0 <= page < self.p.n_pages else None

    def each_row(self):
        """(row, sequence, position) of every row that belongs to a sequence."""
        for s in range(len(self.pairs)):
            r0, r1 = int(self.start[s]), int(self.start[s + 1])
            n = int(self.len[s])
            for r in range(r0, r1):
                yield r, s, n - (r1 - r0) + (r - r0)

    def device(self):
        """Positional arguments (pools, table, seq_len, row_start) and scales on the GPU."""
        def up(t):
            return t.view(torch.uint8).cuda().view(t.dtype) if t.dtype == torch.float8_e4m3fn else t.cuda()
        self.dev = [up(self.pool["K"]), up(self.pool["V"]), self.table.cuda(), self.len.cuda(), self.start.cuda()]
        if self.form != gk.PAGES_PLAIN:
            self.dev += [up(self.pool["Ks"]), up(self.pool["Vs"])]
        return self.dev

    def attend(self, Q, scale=None):
        """(out, lse, bound) in 64 bits; rows of no sequence are NaN.  `bound`: how far an implementation may be off that
        holds logits, weights and sums in 32 bits and, with bf16 rows, rounds the weights to bf16 for the product."""
        c = scale or 1 / math.sqrt(self.d)
        u = 2.0 ** -24
        k, v, q = self.values("K"), self.values("V"), Q.double()
        out = torch.full((self.rows, self.H * self.G, self.d), math.nan, dtype=torch.float64)
        bound = torch.zeros_like(out)
        lse = torch.full((self.rows, self.H * self.G), math.nan, dtype=torch.float64)
        lse_bound = torch.zeros_like(lse)
        for r, s, pos in self.each_row():
            cells = [c for c in (self.place(s, j) for j in range(min(pos + 1, self.table.shape[1] * self.ps))) if c]
            if not cells:
                out[r], lse[r] = 0.0, -math.inf
                continue
            page, at = torch.tensor(cells).T
            for h in range(self.H * self.G):
                kk, vv = k[page, h // self.G, at], v[page, h // self.G, at]
                x = kk @ q[r, h] * c
                w = torch.softmax(x, 0)
                out[r, h] = w @ vv
                lse[r, h] = torch.logsumexp(x, 0)
                # a 32-bit product of d terms, its scales and the subtraction of the maximum
                off = (self.d + 8) * u * float((kk.abs() @ q[r, h].abs()).max()) * c
                terms = (len(cells) + self.d + 64) * u                   # sums of positive terms, a few ulp of the exponential
                weights = half_step(torch.bfloat16) if self.dtype == gk.BF16 else 0.0
                mass = w @ vv.abs()
                bound[r, h] = mass * (weights + 4 * off + 4 * terms) + out[r, h].abs() * half_step(TORCH[self.dtype])
                lse_bound[r, h] = 2 * off + 2 * terms + abs(float(lse[r, h])) * 8 * u
        return out, lse, bound, lse_bound


def check_attend(b, Q, got, lse=None, scale=None):
    out, want_lse, bound, lse_bound = b.attend(Q, scale)
    mine = ~out.isnan()
    got = got.double().cpu()
    assert torch.isfinite(got[mine]).all()
    # (2^-100: results next to nothing are not rounded relative to themselves)
    worst = ((got - out).abs() / (bound + 2.0 ** -100))[mine]
    assert worst.numel() == 0 or float(worst.max()) <= 1.0, f"off by {float(worst.max()):.2f} of what rounding allows"
    if lse is not None:
        lse = lse.double().cpu()
        ok = ~want_lse.isnan()
        none = want_lse == -math.inf
        assert torch.equal(lse[none], want_lse[none])
        assert ((lse - want_lse).abs() <= lse_bound)[ok & ~none].all()
