"""Pages dealt to sequences on the device, against the definition (GPU)."""
import random

import pytest
import torch

from paper_2509_00388_amd import binding as gk
from tests import more_util as mu

pytestmark = pytest.mark.gpu


def say(msg):
    print(msg, flush=True)


class Turn:
    """A pool of pages dealt at random to sequences of these lengths."""

    def __init__(self, had, ps, table_pages, spare, seed=0):
        g = torch.Generator().manual_seed(seed)
        up = [-(-h // ps) for h in had]
        pages = sum(up) + spare
        order = torch.randperm(pages, generator=g).int()
        self.ps, self.had = ps, list(had)
        self.table = torch.randint(0, pages, (len(had), table_pages), generator=g).int()      # (unused entries name some page)
        at = 0
        for s, n in enumerate(up):
            self.table[s, :n] = order[at:at + n]
            at += n
        self.stack = torch.full((pages,), 12345, dtype=torch.int32)
        self.stack[:spare] = order[at:]
        self.n_free = spare

    def params(self, n_rows, max_rows=0):
        return gk.PagedParams(n_kv_heads=1, n_q_heads=1, head_dim=16, page_tokens=self.ps, n_pages=self.stack.numel(), n_seqs=len(self.had),
                              table_pages=self.table.shape[1], n_rows=n_rows, max_rows=max_rows)

    def check(self, new, keep=None, n_rows=None, max_rows=0, in_place=False, maps=True):
        """The call against the definition; what it leaves becomes this state."""
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        n_rows = sum(max(n, 0) for n in new) if n_rows is None else n_rows
        p = self.params(n_rows, max_rows)
        want = mu.assigned(keep or [None] * len(new), new, self.had, self.table, self.stack, self.n_free, self.ps, n_rows, max_rows)
        had, free, table, stack = i32(self.had), i32([self.n_free]), self.table.cuda(), self.stack.cuda()
        pos, slot = (torch.full((n_rows,), -7, dtype=torch.int32, device="cuda") if maps else None for _ in range(2))
        ws = torch.randint(0, 256, (gk.graphkv_assign_workspace_bytes(p),), dtype=torch.uint8, device="cuda")
        out = dict(seq_len=had, free_after=free) if in_place else {}
        length, after, start = gk.graphkv_cache_assign(p, i32(new), had, table, stack, free, keep=i32(keep) if keep else None, positions=pos,
                                                       slots=slot, ws=ws, **out)
        got = (length, table, stack, after, start, pos, slot)
        for name, x, y in zip(("seq_len", "table", "free_pages", "free_after", "row_start", "positions", "slots"), got, want):
            assert x is None or torch.equal(x.cpu(), y), name
        self.had, self.table, self.stack, self.n_free = want[0].tolist(), want[1], want[2], int(want[3])
        return want


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n_seqs,ps,most", [(1, 16, 400), (3, 1, 9), (64, 16, 700), (200, 4, 60), (256, 128, 900), (257, 16, 100), (1000, 16, 70),
                                            (1024, 2, 9), (1025, 16, 80), (2500, 8, 50), (2048, 16, 40), (2049, 16, 20), (4096, 4, 12),
                                            (3000, 4, 90), (4097, 16, 30), (9000, 8, 20)])
def test_turns(n_seqs, ps, most, in_place):
    """Turns of a scheduler: prompts, single tokens, drafts, sequences that are cut or end, pages that run out."""
    say(f"turns n_seqs={n_seqs} ps={ps} in_place={in_place}")
    rng = random.Random(n_seqs + ps)
    had = [rng.choice([0, 1, ps, rng.randint(0, most)]) for _ in range(n_seqs)]
    t = Turn(had, ps, -(-most // ps) + 3, spare=2 + n_seqs // 3, seed=n_seqs)
    for turn in range(6):
        new = [rng.choice([0, 1, 1, 1, 5, rng.randint(0, most)]) for _ in range(n_seqs)]
        keep = [rng.choice([h, h, h, h - 1, 0, h // 2, h + 5]) for h in t.had] if turn % 2 else None
        room = sum(new)
        n_rows = [room, room + 17, max(room - most, 0), room, room + 5000, room // 2][turn]
        t.check(new, keep, n_rows, in_place=in_place, maps=turn != 3)


def test_taken_back():
    """A call that cuts what another added leaves stack and lengths as they were, and what is added again gets the same pages."""
    say("taken back")
    t = Turn([5, 0, 90, 33, 16], 16, 30, spare=40)
    before, stack = list(t.had), t.stack.clone()
    grown = t.check([100, 33, 1, 0, 17])
    assert grown[0].tolist() == [105, 33, 91, 33, 33]
    back = t.check([0] * 5, keep=before)
    assert back[0].tolist() == before and torch.equal(t.stack[:40], stack[:40]) and t.n_free == 40
    again = t.check([100, 33, 1, 0, 17])
    assert torch.equal(again[1], grown[1]) and torch.equal(again[6], grown[6])


@pytest.mark.parametrize("n_seqs", [40, 1500, 4000, 5000])
def test_refusals(n_seqs):
    """Sequences that ask for more than their table, max_rows, the rows or the free pages hold; later ones that ask for less."""
    say(f"refusals n_seqs={n_seqs}")
    ps, W = 8, 5
    had = [(7 * s) % 31 for s in range(n_seqs)]
    new = [1] * n_seqs
    new[3], new[9], new[11], new[20] = 41, 2 ** 31 - 1, -5, 2 ** 31 - 1 - 40
    Turn(had, ps, W, spare=n_seqs, seed=1).check(new, n_rows=n_seqs + 60, max_rows=40)
    Turn(had, ps, W, spare=n_seqs, seed=2).check(new, n_rows=n_seqs + 60)
    Turn(had, ps, W, spare=n_seqs // 16, seed=3).check([3] * n_seqs, n_rows=3 * n_seqs + 1)      # pages run out on the way
    Turn(had, ps, W, spare=0, seed=4).check([3] * n_seqs, n_rows=3 * n_seqs + 1)
    Turn(had, ps, W, spare=n_seqs, seed=5).check([3] * n_seqs, n_rows=n_seqs)                     # rows do
    Turn(had, ps, W, spare=n_seqs, seed=6).check([3] * n_seqs, n_rows=0)
    Turn(had, ps, W, spare=n_seqs, seed=7).check([0] * n_seqs, keep=[0] * n_seqs, n_rows=4)       # all end


def test_long_prompts():
    """Rows and pages far beyond a workgroup's threads, in one sequence and beside others; rows told by either kernel."""
    say("long prompts")
    Turn([1], 64, 3000, spare=3000).check([150001], keep=[0], n_rows=150100)
    Turn([100] * 70, 16, 2100, spare=9000).check([1] * 30 + [31000] + [1] * 38 + [4096], n_rows=40000)
    Turn([10] * 5, 1, 5000, spare=9000).check([4000, 1, 1, 70, 24], n_rows=4096)
    Turn([10] * 5, 1, 5000, spare=9000).check([4000, 1, 1, 70, 25], n_rows=4097)
    Turn([60000] * 3, 16, 4000, spare=1).check([1, 0, 9], keep=[0, 60000, 17])      # thousands of pages come back


def test_arrays_of_any_content():
    """Lengths, page numbers and counts outside their ranges: nothing outside the arrays is touched, and what is stated holds."""
    say("arrays of any content")
    worst = [-2 ** 31, -1, 0, 1, 2 ** 30, 2 ** 31 - 1]
    for n_seqs in (6, 1030, 3000, 4100):
        t = Turn([20] * n_seqs, 4, 9, spare=50, seed=n_seqs)
        t.had = [worst[s % 6] for s in range(n_seqs)]
        keep = [worst[(s // 2) % 6] for s in range(n_seqs)]
        new = [worst[(s // 3) % 6] if s % 5 == 0 else 1 for s in range(n_seqs)]
        for n_free in (-3, 7, 2 ** 31 - 1):
            i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
            p = t.params(700)
            # (a guard on both sides of every array that is written)
            outs = {n: torch.full((c + 64,), -7, dtype=torch.int32, device="cuda") for n, c in
                    (("seq_len", n_seqs), ("free_after", 1), ("row_start", n_seqs + 1), ("positions", 700), ("slots", 700))}
            table, stack = (torch.full((x.numel() + 64,), -7, dtype=torch.int32, device="cuda") for x in (t.table, t.stack))
            table[32:-32], stack[32:-32] = t.table.flatten().cuda(), t.stack.cuda()
            views = {n: x[32:-32] for n, x in outs.items()}
            gk.graphkv_cache_assign(p, i32(new), i32(t.had), table[32:-32], stack[32:-32], i32([n_free]), keep=i32(keep), **views)
            for x in list(outs.values()) + [table, stack]:
                assert (x[:32] == -7).all() and (x[-32:] == -7).all()
            length, start = views["seq_len"].cpu(), views["row_start"].cpu()
            assert ((length >= 0) & (length <= 36)).all() and start[0] == 0 and (start.diff() >= 0).all() and start[-1] <= 700
            assert 0 <= int(views["free_after"]) <= t.stack.numel()


def test_nothing_to_assign():
    say("nothing to assign")
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    p = gk.PagedParams(n_kv_heads=1, n_q_heads=1, head_dim=16, page_tokens=16, n_pages=9, n_seqs=0, table_pages=3, n_rows=5)
    pos, free = torch.full((5,), -7, dtype=torch.int32, device="cuda"), i32(4)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    length, after, start = gk.graphkv_cache_assign(p, none, none, none.view(0, 3), torch.arange(9, dtype=torch.int32, device="cuda"), free, positions=pos)
    assert length.numel() == 0 and after.tolist() == [4] and start.tolist() == [0] and (pos == -1).all()


@pytest.mark.parametrize("n_seqs", [50, 1400, 2100, 4500])
def test_captured_turns(n_seqs):
    """A captured turn, replayed with other lengths, with eager work between: the state that the definition gives."""
    say(f"captured turns n_seqs={n_seqs}")
    rng = random.Random(5)
    t = Turn([rng.randint(0, 90) for _ in range(n_seqs)], 16, 40, spare=3 * n_seqs)
    n_rows = 3 * n_seqs + 9
    p = t.params(n_rows)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    had, free, table, stack = i32(t.had), i32([t.n_free]), t.table.cuda(), t.stack.cuda()
    new, keep, start = i32([0] * n_seqs), i32(t.had), i32([0] * (n_seqs + 1))
    pos, slot = (torch.zeros(n_rows, dtype=torch.int32, device="cuda") for _ in range(2))
    ws = gk.alloc_assign_workspace(p)

    def call():
        gk.graphkv_cache_assign(p, new, had, table, stack, free, keep=keep, seq_len=had, free_after=free, row_start=start, positions=pos,
                                slots=slot, ws=ws)
    call()      # (nothing changes: no new rows)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for n in range(4):
        asks = [rng.choice([0, 1, 1, 2, 3]) for _ in range(n_seqs)]
        keeps = [rng.choice([h, h, h // 2]) for h in t.had]
        new.copy_(i32(asks))
        keep.copy_(i32(keeps))
        graph.replay()
        want = mu.assigned(keeps, asks, t.had, t.table, t.stack, t.n_free, t.ps, n_rows, 0)
        for x, y in zip((had, table, stack, free, start, pos, slot), want):
            assert torch.equal(x.cpu(), y), n
        t.had, t.table, t.stack, t.n_free = want[0].tolist(), want[1], want[2], int(want[3])
        torch.ones(100, device="cuda").sum().item()


def test_binding_refuses_wrong_tensors():
    say("wrong tensors")
    t = Turn([5, 6], 16, 3, spare=4)
    p = t.params(9)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    good = [i32(1, 1), i32(5, 6), t.table.cuda(), t.stack.cuda(), i32(4)]
    for i, bad in ((0, i32(1)), (0, good[0].long()), (1, good[1].cpu()), (2, good[2][:, :2]), (2, t.table), (3, good[3][:-1]), (4, None)):
        args = list(good)
        args[i] = bad
        with pytest.raises(gk.GraphKVError):
            gk.graphkv_cache_assign(p, *args)
    for kw in (dict(keep=i32(1)), dict(seq_len=i32(1)), dict(row_start=i32(1, 1)), dict(positions=i32(1)), dict(slots=torch.zeros(9, device="cuda"))):
        with pytest.raises(gk.GraphKVError):
            gk.graphkv_cache_assign(p, *good, **kw)
    torch.cuda.synchronize()
