"""Batches for the tests of pages in blocks, of attention over another sequence's states and of pages dealt on the device, and
these operators' definitions on the CPU."""
import torch

from paper_2509_00388_amd import binding as gk
from tests import paged_util as pu

BLOCKS = [gk.PAGES_FP8_BLOCKS, gk.PAGES_INT8_BLOCKS]
ROW_FORM = {gk.PAGES_FP8_BLOCKS: gk.PAGES_FP8, gk.PAGES_INT8_BLOCKS: gk.PAGES_INT8}


def codes(x, scale, form):
    """Codes (the values that they stand for before the scale) of values x with these scales, in 64 bits."""
    y = torch.where(scale > 0, x.double() / torch.where(scale > 0, scale, 1.0).double(), 0.0)
    if ROW_FORM.get(form, form) == gk.PAGES_INT8:
        return y.round().clamp(-127, 127)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(y / step) * step


def scale_of(x, form):
    """The scale that rows with these largest magnitudes x [..., values] have, in 64 bits."""
    return pu.encode(x, ROW_FORM.get(form, form))[1]


def stored(code, form):
    return code.to(torch.int8) if ROW_FORM.get(form, form) == gk.PAGES_INT8 else code.float().to(torch.float8_e4m3fn)


class Batch(pu.Batch):
    """pu.Batch with pages in blocks of `block` tokens, or whose rows see all of their sequence (`cross`)."""

    def __init__(self, pairs, form=gk.PAGES_PLAIN, block=16, cross=False, **kw):
        self.block, self.cross = block, cross
        super().__init__(pairs, form=form, **kw)
        if form in BLOCKS:
            self.p.scale_tokens = block

    def set_pool(self, n, x):
        if self.form not in BLOCKS:
            return super().set_pool(n, x)
        y = x.double().reshape(*x.shape[:2], self.ps // self.block, self.block * self.d)
        scale = scale_of(y, self.form)
        self.pool[n] = stored(codes(y, scale[..., None], self.form).reshape(x.shape), self.form)
        self.pool[n + "s"] = scale.float()

    def values(self, n):
        if self.form not in BLOCKS:
            return super().values(n)
        return self.pool[n].double() * self.pool[n + "s"].double().repeat_interleave(self.block, 2)[..., None]

    def each_row(self):
        for r, s, pos in super().each_row():
            yield r, s, min(int(self.len[s]), self.table.shape[1] * self.ps) - 1 if self.cross else pos


def written(b, K, V):
    """What the pools of b hold after its rows are written, by the definition: position by position, a block's scale never less
    than before, earlier codes rounded again where it grows."""
    want = {n: t.clone() for n, t in b.pool.items()}
    raw = lambda t: t.view(torch.uint8)  # noqa: E731
    for s in range(len(b.pairs)):
        r0, n, length = int(b.start[s]), int(b.start[s + 1]) - int(b.start[s]), int(b.len[s])
        first = max(0, length - n)
        for begin in range(first // b.block * b.block, length, b.block):
            cell = b.place(s, begin)
            if cell is None or length <= begin:
                continue
            page, at = cell
            lo, hi = max(first, begin), min(begin + b.block, length)
            if lo >= hi:
                continue
            rows = slice(r0 + lo - (length - n), r0 + hi - (length - n))
            for name, x in (("K", K), ("V", V)):
                new = x[rows].double().transpose(0, 1)                                   # [heads, tokens, d]
                before = want[name + "s"][page, :, at // b.block].double() if lo > begin else torch.zeros(b.H, dtype=torch.float64)
                after = torch.maximum(before, scale_of(new.reshape(b.H, -1), b.form))
                grown = after > before
                old = want[name][page, :, at:at + lo - begin].double() * before[:, None, None]
                again = stored(codes(old, after[:, None, None], b.form), b.form)
                keep = raw(want[name])[page, :, at:at + lo - begin]
                raw(want[name])[page, :, at:at + lo - begin] = torch.where(grown[:, None, None], raw(again), keep)
                raw(want[name])[page, :, at + lo - begin:at + hi - begin] = raw(stored(codes(new, after[:, None, None], b.form), b.form))
                want[name + "s"][page, :, at // b.block] = after.float()
    return want


def assigned(keep, new, had, table, stack, n_free, ps, n_rows, max_rows):
    """Pages dealt one sequence after the other, as the header words it.  Lists and tensors are left as they are; returns
    (seq_len, table, stack, n_free, row_start, positions, slots)."""
    table, stack = table.clone(), stack.clone()
    pages, W = stack.numel(), table.shape[1]
    up = lambda t: -(-t // ps)  # noqa: E731
    n_free = min(max(n_free, 0), pages)
    had = [min(max(h, 0), W * ps) for h in had]
    kept = [h if k is None else min(max(k, 0), h) for k, h in zip(keep, had)]
    new = [max(n, 0) for n in new]
    want = [k + n for k, n in zip(kept, new)]
    ok, asked = [], 0
    for n, w in zip(new, want):
        fits = n <= (max_rows or n_rows) and w <= W * ps
        asked += n if fits else 0
        ok.append(fits and (n == 0 or asked <= n_rows))
    back = [int(p) for s in range(len(had)) if ok[s] for p in table[s, up(want[s]):up(had[s])]]
    free = stack[:n_free].tolist() + back[::-1]
    stack[:len(free)] = torch.tensor(free, dtype=torch.int32)
    left, short = len(free), False
    for s in range(len(had)):
        need = max(0, up(want[s]) - up(had[s])) if ok[s] else 0
        if need and (short or need > left):
            ok[s], short = False, True
        for i in range(need if ok[s] else 0):
            left -= 1
            table[s, up(had[s]) + i] = stack[left]
    length = [w if o else h for w, o, h in zip(want, ok, had)]
    start = [0]
    for s in range(len(had)):
        start.append(start[-1] + (new[s] if ok[s] else 0))
    pos, slot = [-1] * n_rows, [-1] * n_rows
    for s in range(len(had)):
        for r in range(start[s], start[s + 1]):
            pos[r] = length[s] - start[s + 1] + r
            page = int(table[s, pos[r] // ps])
            slot[r] = page * ps + pos[r] % ps if 0 <= page < pages else -1
    i32 = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    return i32(length), table, stack, i32([left]), i32(start), i32(pos), i32(slot)
