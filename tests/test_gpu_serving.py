"""The calls around a paged cache as a serving loop makes them: pages dealt, rows written in blocks, attention, eviction, and attention
over other states (GPU)."""
import pytest
import torch

from paper_2509_00388_amd import binding as gk
from tests import more_util as mu
from tests import paged_util as pu
from tests.test_gpu_paged import on_gpu, say

pytestmark = pytest.mark.gpu

H, G, D, PS, BLOCK, SEQS, WIDTH, PAGES = 2, 4, 128, 32, 16, 4, 30, 70


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Cache:
    """Pools, tables and free pages of a few sequences."""

    def __init__(self, form, seed=1):
        self.form, self.g = form, torch.Generator("cuda").manual_seed(seed)
        self.pool = [torch.zeros(PAGES, H, PS, D, device="cuda").to(mu.stored(torch.zeros(1), form).dtype) for _ in range(2)]
        self.scales = [torch.zeros(PAGES, H, PS // BLOCK, device="cuda") for _ in range(2)]
        self.table = torch.zeros(SEQS, WIDTH, dtype=torch.int32, device="cuda")
        self.free = torch.randperm(PAGES, generator=self.g, device="cuda").to(torch.int32)
        self.n_free, self.len = i32([PAGES]), i32([0] * SEQS)

    def params(self, rows, most, seqs=SEQS):
        return gk.PagedParams(n_kv_heads=H, n_q_heads=H * G, head_dim=D, page_tokens=PS, n_pages=PAGES, n_seqs=seqs, table_pages=WIDTH, n_rows=rows,
                              max_rows=most, page_format=self.form, scale_tokens=BLOCK)

    def turn(self, new, keep=None):
        """Deals pages; (params, row numbers, positions, slots)."""
        p = self.params(sum(new), max(new))
        pos, slot = (torch.empty(sum(new), dtype=torch.int32, device="cuda") for _ in range(2))
        _, _, start = gk.graphkv_cache_assign(p, i32(new), self.len, self.table, self.free, self.n_free, keep=None if keep is None else i32(keep),
                                              seq_len=self.len, free_after=self.n_free, positions=pos, slots=slot)
        self.check_pages()
        return p, start, pos, slot

    def check_pages(self):
        """Every page belongs to one sequence or is free."""
        n = int(self.n_free)
        held = [int(p) for s in range(SEQS) for p in self.table[s, :-(-int(self.len[s]) // PS)]]
        assert sorted(held + self.free[:n].tolist()) == list(range(PAGES))

    def rows(self, n):
        qkv = torch.randn(n, (G + 2) * H, D, generator=self.g, device="cuda").to(torch.bfloat16)
        return qkv[:, :G * H], qkv[:, G * H:G * H + H], qkv[:, G * H + H:]

    def batch(self, start):
        return (self.table, self.len, start)

    def definition(self, p, start, cross=False):
        b = mu.Batch([(int(start[s + 1] - start[s]), int(self.len[s])) for s in range(SEQS)], form=self.form, block=BLOCK, cross=cross, H=H, G=G, d=D,
                     ps=PS, table_pages=WIDTH)
        b.p, b.table, b.len, b.start, b.rows = p, self.table.cpu(), self.len.cpu(), start.cpu(), p.n_rows
        b.pool = {n: t.cpu() for n, t in zip(("K", "V", "Ks", "Vs"), self.pool + self.scales)}
        return b


@pytest.mark.parametrize("form", mu.BLOCKS)
def test_serving_loop(form):
    say(f"serving loop form={form}")
    c = Cache(form)
    window, budget, length = 16, 150, 700
    for step, (new, keep) in enumerate([([length, 1, 77, 0], None), ([1, 5, 1, 300], None), ([1, 1, 1, 1], None), ([budget, 1, 1, 1], "evict"),
                                        ([1, 1, 1, 1], None), ([1, 0, 90, 2], "end"), ([1, 1, 1, 1], None)]):
        if keep == "evict":
            # the first sequence read back as the eviction pass takes it; what it keeps goes to fewer pages
            n = int(c.len[0])
            rp = c.params(n, n)
            Kc, Vc = (torch.empty(H, n, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            gk.graphkv_cache_read(rp, *c.pool, *c.batch(i32([0] + [n] * SEQS)), *c.scales, K=Kc.transpose(0, 1), V=Vc.transpose(0, 1))
            ep = gk.Params(n_kv_heads=H, n_q_heads=G * H, head_dim=D, n_tokens=n, window=window, pool_kernel=5, budget=budget, n_sources=8, n_neighbors=4,
                           rounds=1)
            Qw = torch.randn(G * H, window, D, generator=c.g, device="cuda").to(torch.bfloat16)
            Ko, Vo, _ = gk.graphkv_compress(ep, Kc, Vc, Qw)
            keep = [0] + c.len.tolist()[1:]
        elif keep == "end":
            keep = c.len.tolist()
            keep[2] = 0
        before = c.len.tolist()
        p, start, pos, slot = c.turn(new, keep)
        assert c.len.tolist() == [(k if keep else b) + n for k, b, n in zip(keep or before, before, new)]
        Q, K, V = c.rows(p.n_rows)
        if step == 3:
            K, V = torch.cat([Ko.transpose(0, 1), K[budget:]]), torch.cat([Vo.transpose(0, 1), V[budget:]])
        gk.graphkv_cache_write(p, K.contiguous(), V.contiguous(), *c.pool, *c.batch(start), *c.scales)
        # what the slots name is what a read gives
        Kr, _ = gk.graphkv_cache_read(p, *c.pool, *c.batch(start), *c.scales)
        page, at = slot.long() // PS, slot.long() % PS
        code = c.pool[0].view(torch.uint8)[page, :, at].view(c.pool[0].dtype).double() * c.scales[0][page, :, at // BLOCK].double()[..., None]
        assert torch.equal(Kr, code.to(torch.bfloat16))
        seq = torch.searchsorted(start[1:], torch.arange(p.n_rows, device="cuda"), right=True)
        assert torch.equal(pos, (c.len[seq] - start[seq + 1] + torch.arange(p.n_rows, device="cuda")).int())
        lse = torch.empty(p.n_rows, H * G, device="cuda")
        out = gk.graphkv_attend(p, Q, *c.pool, *c.batch(start), *c.scales, lse=lse)
        if step != 0:       # (the definition takes a while for long chunks)
            pu.check_attend(c.definition(p, start), Q.cpu(), out, lse)
    # rows of another model part over what the sequences hold
    q = c.params(11, 5)
    start = i32([0, 1, 6, 6, 11])
    Q = c.rows(11)[0]
    lse = torch.empty(11, H * G, device="cuda")
    out = gk.graphkv_cross_attend(q, Q, *c.pool, *c.batch(start), *c.scales, lse=lse)
    pu.check_attend(c.definition(q, start, cross=True), Q.cpu(), out, lse)


@pytest.mark.parametrize("form", mu.BLOCKS)
def test_captured_steps(form):
    """A decoding step as one graph (pages dealt, rows written, attention), replayed with eager work between: the bits of the same steps made
    one by one."""
    say(f"captured steps form={form}")

    def start_of(c):
        p, start, _, _ = c.turn([300, 1, 62, 31])
        _, K, V = c.rows(p.n_rows)
        gk.graphkv_cache_write(p, K, V, *c.pool, *c.batch(start), *c.scales)

    steps = 6
    one, two = Cache(form, 3), Cache(form, 3)
    for c in (one, two):
        start_of(c)
    data = [one.rows(SEQS + 2) for _ in range(steps)]            # (two rows more than sequences: a batch padded to a fixed size)
    asks = [[1, 1, 1, 1], [1, 0, 2, 1], [1, 1, 1, 2], [0, 1, 1, 1], [1, 1, 1, 1], [2, 1, 1, 1]]
    p = one.params(SEQS + 2, 2)
    want = []
    for (Q, K, V), new in zip(data, asks):
        _, _, start = gk.graphkv_cache_assign(p, i32(new), one.len, one.table, one.free, one.n_free, seq_len=one.len, free_after=one.n_free)
        gk.graphkv_cache_write(p, K, V, *one.pool, *one.batch(start), *one.scales)
        out = torch.full((SEQS + 2, H * G, D), -7.0, dtype=torch.bfloat16, device="cuda")
        want.append(gk.graphkv_attend(p, Q, *one.pool, *one.batch(start), *one.scales, out=out))
    Q, K, V = (x.clone() for x in two.rows(SEQS + 2))
    new, start, out, ws = i32([0] * SEQS), i32([0] * (SEQS + 1)), torch.empty_like(want[0]), gk.alloc_attend_workspace(p)

    def step():
        gk.graphkv_cache_assign(p, new, two.len, two.table, two.free, two.n_free, seq_len=two.len, free_after=two.n_free, row_start=start)
        gk.graphkv_cache_write(p, K, V, *two.pool, *two.batch(start), *two.scales)
        gk.graphkv_attend(p, Q, *two.pool, *two.batch(start), *two.scales, out=out, ws=ws)
    step()       # (no new rows: nothing changes)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(steps):
        for to, x in zip((Q, K, V), data[i]):
            to.copy_(x)
        new.copy_(i32(asks[i]))
        out.fill_(-7)
        graph.replay()
        assert torch.equal(out, want[i]), i
        torch.ones(1000, device="cuda").sum().item()
    for x, y in zip(one.pool + one.scales + [one.table, one.len], two.pool + two.scales + [two.table, two.len]):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
