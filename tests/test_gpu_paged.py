"""The paged cache through the C ABI: rows written to pages, read back, attention over them, against their definitions in
64 bits (GPU)."""
import math

import pytest
import torch

from paper_2509_00388_amd import binding as gk
from tests import paged_util as pu

pytestmark = pytest.mark.gpu

FORMS = [gk.PAGES_PLAIN, gk.PAGES_FP8, gk.PAGES_INT8]
TYPES = [gk.BF16, gk.FP32]


def say(msg):
    print(msg, flush=True)


def on_gpu(t):
    """The same values and strides on the GPU."""
    out = torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device="cuda")
    out.copy_(t)
    return out


def bits(t):
    return t.cpu().contiguous().view(torch.uint8)


# ---- write and read ---------------------------------------------------------------------------------

def written(b, K, V):
    """What the pools hold after a write, by the definition."""
    want = {n: t.clone() for n, t in b.pool.items()}
    for n, x in (("K", K), ("V", V)):
        if b.form != gk.PAGES_PLAIN:
            code, scale = pu.encode(x, b.form)
        for r, s, pos in b.each_row():
            cell = b.place(s, pos)
            if cell is None:
                continue
            page, at = cell
            if b.form == gk.PAGES_PLAIN:
                want[n][page, :, at] = x[r]
            else:
                c = code[r].to(torch.int8) if b.form == gk.PAGES_INT8 else code[r].float().to(torch.float8_e4m3fn)
                want[n].view(torch.uint8)[page, :, at] = c.view(torch.uint8)
                want[n + "s"][page, :, at] = scale[r].float()
    return want


def check_write(b, K, V):
    want = written(b, K, V)
    args = b.device()
    gk.graphkv_cache_write(b.p, on_gpu(K), on_gpu(V), *args)
    names = ["K", "V"] + (["Ks", "Vs"] if b.form != gk.PAGES_PLAIN else [])
    for n, got in zip(names, args[:2] + args[5:]):
        assert torch.equal(bits(got), bits(want[n])), f"pool {n}"
    return args


def check_read(b, args, by_head=False):
    if by_head:
        K, V = (torch.full((b.H, b.rows, b.d), -7.0, dtype=b.p.torch_dtype, device="cuda").transpose(0, 1) for _ in range(2))
    else:
        K, V = (torch.full((b.rows, b.H, b.d), -7.0, dtype=b.p.torch_dtype, device="cuda") for _ in range(2))
    gk.graphkv_cache_read(b.p, *args, K=K, V=V)
    pools = [t.cpu() for t in args[:2]]
    scales = [t.cpu() for t in args[5:]] or [None, None]
    for got, pool, scale in zip((K.cpu(), V.cpu()), pools, scales):
        want = torch.full((b.rows, b.H, b.d), -7.0).to(b.p.torch_dtype)
        for r, s, pos in b.each_row():
            cell = b.place(s, pos)
            if cell is None:
                want[r] = 0
                continue
            x = pool.view(torch.uint8)[cell[0], :, cell[1]].view(pool.dtype) if b.form == gk.PAGES_FP8 else pool[cell[0], :, cell[1]]
            want[r] = x if scale is None else (x.float() * scale[cell[0], :, cell[1]][:, None]).to(b.p.torch_dtype)
        assert torch.equal(bits(got), bits(want))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("d,H,ps,how", [(64, 2, 16, "packed"), (128, 8, 64, "fused"), (80, 3, 1, "by_head"), (16, 5, 128, "packed"),
                                        (512, 1, 8, "fused"), (256, 7, 32, "by_head")])
def test_rows_written_and_read_back(dtype, form, d, H, ps, how):
    say(f"write and read dtype={dtype} form={form} d={d} H={H} ps={ps} {how}")
    b = pu.Batch([(1, 1), (5, 40), (0, 17), (33, 33), (7, 130)], H=H, d=d, ps=ps, dtype=dtype, form=form, before=2, behind=3,
                 seed=d + H)
    K, V = (b.random_rows(H, by_head=how == "by_head", fused=4 if how == "fused" else 0) for _ in range(2))
    K *= torch.exp(3 * torch.randn(b.rows, H, 1, generator=b.g)).to(K.dtype)
    args = check_write(b, K, V)
    check_read(b, args, by_head=how != "packed")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", [gk.PAGES_FP8, gk.PAGES_INT8])
def test_codes_next_to_borders(dtype, form):
    """Rows whose largest value is a border of the scale, values in the middle of two codes, the least and the largest
    magnitudes, zeros of both signs."""
    say(f"codes next to borders dtype={dtype} form={form}")
    d, H = 64, 4
    b = pu.Batch([(64, 64)], H=H, d=d, ps=16, dtype=dtype, form=form, seed=3)
    K, V = b.random_rows(H), b.random_rows(H)
    most = 127.0 if form == gk.PAGES_INT8 else 448.0
    for r in range(64):
        top = most * 2.0 ** (r % 7 - 3)
        K[r] = (torch.randint(-256, 257, (H, d), generator=b.g) * 0.5 * 2.0 ** (r % 7 - 3)).clamp(-top, top)   # many exact middles
        K[r, :, 5] = top
        V[r, :, 7] = [1.0, 448.0, 449.0, 448.0 * 2.0 ** -20, 450.0, 3e38, 1.75, 2.0 ** -99][r % 8]
        V[r, :, 8] = V[r, :, 7] / 2
        V[r, :, 9] = -V[r, :, 7]
    V[9] = 0.0
    V[10] = -0.0
    V[11] = 2.0 ** -101
    check_write(b, K, V)


def test_integer_codes_are_rounded_once():
    """Products of integer codes and scales of all 24 bits that lie next to the middle of two bf16 numbers: to 32 bits they round onto it."""
    say("integer codes rounded once")
    H, d, ps, n = 4, 64, 32, 512
    b = pu.Batch([(n, n)], H=H, d=d, ps=ps, form=gk.PAGES_INT8, seed=21)
    code = torch.randint(3, 128, (b.p.n_pages, H, ps), generator=b.g)
    middle = (257 + 2 * torch.randint(0, 128, code.shape, generator=b.g)).double() / 512 * 2.0 ** torch.randint(-20, 20, code.shape, generator=b.g)
    for name in "KV":
        b.pool[name] = torch.randint(-127, 128, (b.p.n_pages, H, ps, d), generator=b.g).to(torch.int8)
        b.pool[name][..., 0::4] = code[..., None].to(torch.int8)
        b.pool[name][..., 2::8] = -code[..., None].to(torch.int8)
        b.pool[name + "s"] = (middle / code).float()
    K, V = gk.graphkv_cache_read(b.p, *b.device())
    twice = 0
    for got, name in ((K, "K"), (V, "V")):
        for r, s, pos in b.each_row():
            page, at = b.place(s, pos)
            x = b.pool[name][page, :, at].double() * b.pool[name + "s"][page, :, at].double()[:, None]   # exact
            m, e = torch.frexp(x)
            want = torch.ldexp(torch.round(m * 256) / 256, e)   # 8 bits, ties to even
            assert torch.equal(got[r].cpu().double(), want), (name, r)
            twice += int((x.float().to(torch.bfloat16).double() != want).sum())
    assert twice > 1000


def test_rows_without_a_place():
    """Page numbers outside the pool, rows that come before a sequence's first token, lengths beyond the table: not written,
    read as zeros; nothing else changes."""
    say("rows without a place")
    for form in FORMS:
        b = pu.Batch([(6, 30), (5, 3), (4, 50), (3, 20)], H=3, d=32, ps=8, dtype=gk.BF16, form=form, before=1, behind=1, seed=9)
        b.table[0, 3] = -1
        b.table[2, 5] = b.p.n_pages
        b.table[2, 6] = 2 ** 31 - 1
        K, V = b.random_rows(3), b.random_rows(3)
        args = check_write(b, K, V)
        check_read(b, args)
        # a length beyond the table is cut to it
        b.len[3] = 10 ** 9
        args[3] = b.len.cuda()
        b.len[3] = b.table.shape[1] * b.ps
        check_read(b, args)
        # row numbers that do not ascend, or lie outside the tensors: whatever is read, no row outside a sequence is touched
        for odd in ([-5, 3, 3, 900, 2], [7, 2, 1, 0, -1], [19, 19, 19, 19, 19]):
            args[4] = torch.tensor(odd, dtype=torch.int32, device="cuda")
            gk.graphkv_cache_write(b.p, on_gpu(K), on_gpu(V), *args)
            gk.graphkv_cache_read(b.p, *args)
            gk.graphkv_attend(b.p, on_gpu(K), *args)
        torch.cuda.synchronize()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pairs,G", [([(6, 30), (5, 90), (4, 50), (3, 20)], 2), ([(150, 200), (60, 100), (3, 40), (20, 20)], 2), ([(20, 90), (9, 9), (16, 70), (30, 40)], 4)])
def test_row_numbers_outside_the_tensors(dtype, form, pairs, G):
    """Row numbers that do not ascend or lie outside the tensors, as the header says what becomes of them: cut to the tensors and to
    the most rows of a sequence.  Rows and places of no sequence keep what they hold; what exactly one sequence owns is right."""
    say(f"row numbers dtype={dtype} form={form} {pairs}")
    d, H = 32, 2
    b = pu.Batch(pairs, H=H, G=G, d=d, ps=8, dtype=dtype, form=form, before=1, behind=2, seed=31)
    rows, most = b.rows, b.p.max_rows
    K, V, Q = b.random_rows(H), b.random_rows(H), b.random_rows(H * G)
    k, v, c, u = b.values("K"), b.values("V"), 1 / math.sqrt(d), 2.0 ** -24
    for start in ([-5, 3, 3, 900, 2], [7, 2, 1, 0, -1], [rows] * 5, [0, rows, 5, rows, 2 ** 31 - 1], [-2 ** 31, rows // 2, rows // 3, rows, 0],
                  [rows - 1, 4, rows + 7, 9, rows - 2]):
        b.start = torch.tensor(start, dtype=torch.int32)
        spans = []
        for s in range(4):
            r0 = min(max(start[s], 0), rows)
            spans.append((r0, min(min(max(start[s + 1], r0), rows) - r0, most)))
        # write and read go by the row: its sequence is the number of those that end at or before it
        owner = [sum(start[s + 1] <= r for s in range(4)) for r in range(rows)]
        cells = {}
        for r in range(rows):
            s = owner[r]
            if s < 4 and spans[s][0] <= r < sum(spans[s]):
                cells[r] = b.place(s, int(b.len[s]) - spans[s][1] + r - spans[s][0])
        args = b.device()
        gk.graphkv_cache_write(b.p, on_gpu(K), on_gpu(V), *args)
        for i, (name, x) in enumerate((("K", K), ("V", V))):
            want = b.pool[name].clone()
            code, scale = (x, None) if form == gk.PAGES_PLAIN else pu.encode(x, form)
            code = code.to(torch.int8) if form == gk.PAGES_INT8 else code.float().to(torch.float8_e4m3fn) if form == gk.PAGES_FP8 else code
            want_scale = None if scale is None else b.pool[name + "s"].clone()
            for r, cell in cells.items():
                if cell:
                    want.view(torch.uint8)[cell[0], :, cell[1]] = code[r].contiguous().view(torch.uint8)
                    if scale is not None:
                        want_scale[cell[0], :, cell[1]] = scale[r].float()
            assert torch.equal(bits(args[i]), bits(want)), (start, name)
            assert scale is None or torch.equal(bits(args[5 + i]), bits(want_scale)), (start, name)
        args = b.device()
        back = [torch.full((rows, H, d), -7.0, dtype=b.p.torch_dtype, device="cuda") for _ in range(2)]
        gk.graphkv_cache_read(b.p, *args, K=back[0], V=back[1])
        for got, values in zip(back, (k, v)):
            want = torch.full((rows, H, d), -7.0).to(b.p.torch_dtype)
            for r, cell in cells.items():
                want[r] = values[cell[0], :, cell[1]].to(b.p.torch_dtype) if cell else 0
            assert torch.equal(got.cpu(), want), start
        out = torch.full((rows, H * G, d), -7.0, dtype=b.p.torch_dtype, device="cuda")
        lse = torch.full((rows, H * G), -7.0, device="cuda")
        ws = torch.randint(0, 256, (gk.graphkv_attend_workspace_bytes(b.p),), dtype=torch.uint8, device="cuda")
        gk.graphkv_attend(b.p, on_gpu(Q), *args, out=out, lse=lse, ws=ws)
        out, lse = out.cpu().double(), lse.cpu()
        for r in range(rows):
            mine = [s for s in range(4) if spans[s][0] <= r < sum(spans[s])]
            if not mine:
                assert (out[r] == -7).all() and (lse[r] == -7).all(), (start, r)
            if len(mine) != 1:
                continue
            s, = mine
            pos = int(b.len[s]) - spans[s][1] + r - spans[s][0]
            seen = [b.place(s, j) for j in range(pos + 1)]
            if not seen:
                assert (out[r] == 0).all() and (lse[r] == -math.inf).all(), (start, r)
                continue
            page, at = torch.tensor(seen).T
            for h in range(H * G):
                kk, vv = k[page, h // G, at], v[page, h // G, at]
                q = Q[r, h].double()
                w = torch.softmax(kk @ q * c, 0)
                off = (d + 8) * u * float((kk.abs() @ q.abs()).max()) * c
                half = pu.half_step(torch.bfloat16) if dtype == gk.BF16 else 0.0
                allow = (w @ vv.abs()) * (half + 4 * off + 4 * (len(seen) + d + 64) * u) + (w @ vv).abs() * pu.half_step(b.p.torch_dtype)
                assert ((out[r, h] - w @ vv).abs() <= allow).all(), (start, r, h)


def test_long_offsets():
    """Places beyond 2^32 bytes of a pool."""
    say("long offsets")
    H, d, ps, pages = 8, 128, 64, 40000
    b = pu.Batch([(40, 40)], H=H, d=d, ps=ps, dtype=gk.BF16, seed=1)
    b.p.n_pages = pages
    pool = [torch.zeros(pages, H, ps, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    assert (pages - 1) * H * ps * d * 2 > 2 ** 32   # where the last page begins
    K, V = b.random_rows(H), b.random_rows(H)
    Q = b.random_rows(H)
    b.p.n_q_heads = H
    outs = []
    for page in (3, pages - 1):
        b.table[0, 0] = page
        args = [*pool, b.table.cuda(), b.len.cuda(), b.start.cuda()]
        gk.graphkv_cache_write(b.p, on_gpu(K), on_gpu(V), *args)
        k, v = gk.graphkv_cache_read(b.p, *args)
        assert torch.equal(bits(k), bits(K)) and torch.equal(bits(v), bits(V))
        assert torch.equal(bits(pool[0][page, :, :40].transpose(0, 1)), bits(K))
        outs.append(gk.graphkv_attend(b.p, on_gpu(Q), *args))
    assert torch.equal(outs[0], outs[1])


@pytest.mark.parametrize("impl", [gk.IMPL_AUTO, gk.IMPL_GENERIC])
def test_most_rows(impl):
    """Sequences that lie at the end of the most rows that a call takes: theirs are written, read and attended to, no other is
    touched."""
    say("most rows")
    rows, d = (1 << 24) - 1, 8
    p = gk.PagedParams(n_kv_heads=1, n_q_heads=1, head_dim=d, page_tokens=4, n_pages=6, n_seqs=2, table_pages=3, n_rows=rows,
                       max_rows=3, impl=impl)
    table = torch.tensor([[4, 1, 0], [2, 5, 3]], dtype=torch.int32, device="cuda")
    length = torch.tensor([2, 3], dtype=torch.int32, device="cuda")
    start = torch.tensor([rows - 5, rows - 3, rows], dtype=torch.int32, device="cuda")
    K, V, Q = (torch.zeros(rows, 1, d, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    g = torch.Generator().manual_seed(11)
    for t in (K, V, Q):
        t[-5:] = torch.randn(5, 1, d, generator=g).to(torch.bfloat16).cuda()
    pools = [torch.full((6, 1, 4, d), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    gk.graphkv_cache_write(p, K, V, *pools, table, length, start)
    for pool, x in zip(pools, (K, V)):
        want = torch.full((6, 1, 4, d), 9.0, dtype=torch.bfloat16)
        want[4, 0, :2], want[2, 0, :3] = x[-5:-3, 0].cpu(), x[-3:, 0].cpu()
        assert torch.equal(bits(pool), bits(want))
    back = [torch.full((rows, 1, d), -7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    gk.graphkv_cache_read(p, *pools, table, length, start, K=back[0], V=back[1])
    out = torch.full((rows, 1, d), -7.0, dtype=torch.bfloat16, device="cuda")
    gk.graphkv_attend(p, Q, *pools, table, length, start, out=out)
    for t in (*back, out):
        assert bool((t[:-5] == -7).all())
    assert torch.equal(bits(back[0][-5:]), bits(K[-5:])) and torch.equal(bits(back[1][-5:]), bits(V[-5:]))
    for a, n in ((rows - 5, 2), (rows - 3, 3)):
        k, v, q = (t[a:a + n, 0].cpu().double() for t in (K, V, Q))
        x = (q @ k.T / math.sqrt(d)).masked_fill(torch.ones(n, n).triu(1).bool(), -math.inf)
        want = torch.softmax(x, 1) @ v
        # weights and output are rounded to bf16, half a step each (and 32-bit sums of at most 8 and 3 terms, far below)
        assert bool(((out[a:a + n, 0].cpu().double() - want).abs() <= 2 ** -7 * 1.01 * v.abs().max()).all())


# ---- attention --------------------------------------------------------------------------------------

def run_attend(b, Q, **kw):
    args = b.device()
    out = torch.full((b.rows, b.H * b.G, b.d), -7.0, dtype=b.p.torch_dtype, device="cuda")
    lse = torch.full((b.rows, b.H * b.G), -7.0, device="cuda")
    ws = torch.randint(0, 256, (gk.graphkv_attend_workspace_bytes(b.p),), dtype=torch.uint8, device="cuda")
    gk.graphkv_attend(b.p, on_gpu(Q), *args, out=out, lse=lse, ws=ws, **kw)
    outside = torch.ones(b.rows, dtype=torch.bool)
    for r, _, _ in b.each_row():
        outside[r] = False
    assert (out.cpu()[outside] == -7).all() and (lse.cpu()[outside] == -7).all()
    return out, lse


SHAPES = [
    # single tokens, few and many tiles, one and several query heads
    dict(pairs=[(1, 1)], H=1, G=1, d=128), dict(pairs=[(1, 129), (1, 31), (1, 1), (1, 512)], H=2, G=4, d=128),
    dict(pairs=[(1, 700), (1, 64)], H=3, G=7, d=64, ps=32), dict(pairs=[(1, 300)] * 5, H=2, G=32, d=80, ps=8),
    # drafts
    dict(pairs=[(8, 100), (3, 3), (1, 250)], H=2, G=4, d=128, ps=64), dict(pairs=[(4, 77)], H=1, G=8, d=64, ps=1),
    # chunks, alone and beside single tokens; blocks that end inside a sequence
    dict(pairs=[(100, 300)], H=2, G=4, d=128), dict(pairs=[(33, 33)], H=3, G=1, d=64, ps=32),
    dict(pairs=[(1, 150), (70, 200), (8, 90), (129, 130)], H=2, G=2, d=128, ps=32),
    dict(pairs=[(19, 260), (0, 50), (50, 50)], H=2, G=7, d=96, ps=128),
    # many sequences of either kind: both kernels
    dict(pairs=[(1, 150), (70, 200), (8, 90), (129, 130), (1, 1), (1, 33), (2, 64), (0, 9), (1, 400)], H=2, G=2, d=128, ps=32),
    dict(pairs=[(1, 90), (30, 60), (2, 90), (1, 0), (1, 7), (1, 33), (5, 64), (3, 2), (40, 100)], H=2, G=7, d=64, ps=2),
    # a token a page, blocks of each size
    dict(pairs=[(150, 200)], H=1, G=2, d=128, ps=1), dict(pairs=[(60, 130)], H=1, G=1, d=80, ps=2), dict(pairs=[(100, 101)], H=2, G=1, d=128, ps=4),
    # other head dimensions
    dict(pairs=[(1, 200), (40, 140)], H=2, G=2, d=256), dict(pairs=[(3, 120)], H=2, G=2, d=160, ps=64),
    dict(pairs=[(2, 90), (20, 60)], H=1, G=2, d=512), dict(pairs=[(1, 100), (45, 45)], H=2, G=1, d=16),
    # a group of more query heads than the kernel for few rows takes
    dict(pairs=[(1, 140)], H=1, G=48, d=64),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_attention(dtype, form, shape):
    say(f"attention dtype={dtype} form={form} {SHAPES[shape]}")
    b = pu.Batch(dtype=dtype, form=form, before=1, behind=2, seed=shape, **SHAPES[shape])
    Q = b.random_rows(b.H * b.G, fused=2 * b.H)
    out, lse = run_attend(b, Q)
    pu.check_attend(b, Q, out, lse)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", FORMS)
def test_attention_scalar_kernel(dtype, form):
    say(f"attention, scalar kernel dtype={dtype} form={form}")
    b = pu.Batch([(1, 400), (30, 300), (4, 2)], H=2, G=2, d=72 if form == gk.PAGES_PLAIN else 80, ps=16, dtype=dtype, form=form,
                 impl=gk.IMPL_GENERIC, before=1, behind=1)
    assert gk.graphkv_attend_workspace_bytes(b.p) == 0
    Q = b.random_rows(4)
    out, lse = run_attend(b, Q)
    pu.check_attend(b, Q, out, lse)


@pytest.mark.parametrize("impl", [gk.IMPL_AUTO, gk.IMPL_GENERIC])
@pytest.mark.parametrize("dtype", TYPES)
def test_attention_of_rows_that_see_nothing(dtype, impl):
    """Sequences without tokens, more rows than tokens, pages that are none: zeros and -infinity."""
    say(f"rows that see nothing dtype={dtype} impl={impl}")
    b = pu.Batch([(1, 0), (5, 2), (60, 20), (1, 40), (40, 90), (2, 33)], H=2, G=2, d=64, ps=8, dtype=dtype, impl=impl, before=1, behind=1)
    b.table[3, :] = -1
    b.table[4, 0] = b.p.n_pages
    b.table[4, 5] = -2 ** 31
    b.table[5, 3] = 10 ** 6
    Q = b.random_rows(4)
    out, lse = run_attend(b, Q)
    pu.check_attend(b, Q, out, lse)
    assert (out.cpu()[1] == 0).all() and (lse.cpu()[1] == -math.inf).all()


@pytest.mark.parametrize("impl", [gk.IMPL_AUTO, gk.IMPL_GENERIC])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pairs,G,d", [([(1, 1)], 4, 64), ([(1, 300), (8, 90)], 4, 128), ([(1, 40), (2, 30)], 2, 256), ([(12, 300), (3, 40)], 4, 128),
                                       ([(30, 200)], 4, 64), ([(90, 400), (30, 60)], 4, 128)])
def test_attention_of_infinite_values(dtype, impl, pairs, G, d):
    """Values that are infinite, at positions that all rows see and that some do: infinities of their sign in the rows that see them and
    in no other place."""
    say(f"infinite values dtype={dtype} impl={impl} {pairs} G={G} d={d}")
    b = pu.Batch(pairs, H=2, G=G, d=d, ps=16, dtype=dtype, impl=impl, before=1, behind=1)
    Q = b.random_rows(2 * G)
    finite = b.pool["V"].clone()
    odd = {}
    for s, (n, length) in enumerate(pairs):
        for j, column, sign in ((0, 3, 1), (length // 3, 20, -1), (length - 1 - n // 2, 40, 1)):
            page, at = b.place(s, j)
            b.pool["V"][page, :, at, column] = sign * math.inf
            finite[page, :, at, column] = 0
            odd[s, column] = (j, sign)
    out, lse = run_attend(b, Q)
    b.pool["V"] = finite
    want, want_lse, bound, lse_bound = b.attend(Q)
    out, lse = out.cpu().double(), lse.cpu().double()
    for r, s, pos in b.each_row():
        rest = torch.ones(d, dtype=torch.bool)
        for (owner, column), (j, sign) in odd.items():
            if owner == s and j <= pos:
                assert (out[r, :, column] == sign * math.inf).all(), (r, s, pos, column)
                rest[column] = False
        assert ((out[r] - want[r]).abs() <= bound[r] + 2.0 ** -100)[:, rest].all(), (r, s, pos)
        assert ((lse[r] - want_lse[r]).abs() <= lse_bound[r]).all(), (r, s, pos)


@pytest.mark.parametrize("impl", [gk.IMPL_AUTO, gk.IMPL_GENERIC])
@pytest.mark.parametrize("dtype", TYPES)
def test_attention_of_logits_of_minus_infinity(dtype, impl):
    """Logits of -infinity weigh nothing; rows that see nothing else have zeros and -infinity, as rows that see nothing."""
    say(f"logits of -infinity dtype={dtype} impl={impl}")
    for pairs, G in (([(1, 300), (8, 90)], 4), ([(12, 300), (3, 40)], 4), ([(90, 400), (30, 60)], 4)):
        b = pu.Batch(pairs, H=2, G=G, d=64, ps=16, dtype=dtype, impl=impl, before=1, behind=1)
        Q = b.random_rows(2 * G)
        Q[:, :, 7] = 1.5
        for j in range(b.pairs[1][1]):
            page, at = b.place(1, j)
            b.pool["K"][page, :, at, 7] = -math.inf
        n = pairs[0][1]
        for j in list(range(0, n // 2)) + [n - 2]:
            page, at = b.place(0, j)
            b.pool["K"][page, :, at, 7] = -math.inf
        out, lse = run_attend(b, Q)
        r0, r1, r2 = b.start.tolist()
        assert (out[r1:r2] == 0).all() and (lse[r1:r2] == -math.inf).all()
        # the first sequence as if those keys were not there
        kept = pu.Batch(pairs, H=2, G=G, d=64, ps=16, dtype=dtype, impl=impl, before=1, behind=1)
        for name in "KV":
            kept.pool[name] = b.pool[name]
        cell = kept.place
        kept.place = lambda s, pos: None if s == 1 or pos < n // 2 or pos == n - 2 else cell(s, pos)
        pu.check_attend(kept, Q, out, lse)


@pytest.mark.parametrize("impl", [gk.IMPL_AUTO, gk.IMPL_GENERIC])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("d", [64, 128])
def test_attention_does_not_see_what_is_hidden(dtype, form, impl, d):
    """Infinities and NaN in the rest of a page, in other pages and at later positions change nothing, bit for bit."""
    say(f"hidden places dtype={dtype} form={form} impl={impl} d={d}")
    b = pu.Batch([(1, 70), (6, 50), (40, 170), (3, 1)], H=2, G=2, d=d, ps=32, dtype=dtype, form=form, impl=impl)
    Q = b.random_rows(4)
    clean, clean_lse = run_attend(b, Q)
    pu.check_attend(b, Q, clean, clean_lse)
    used = torch.zeros(b.p.n_pages, b.ps, dtype=torch.bool)
    for s, (_, n) in enumerate(b.pairs):
        for j in range(n):
            page, at = b.place(s, j)
            used[page, at] = True
    for n in "KV":
        if form == gk.PAGES_PLAIN:
            b.pool[n].transpose(1, 2)[~used] = math.nan
            b.pool[n].transpose(1, 2)[tuple((~used).nonzero()[::3].T)] = math.inf
        else:
            b.pool[n].view(torch.uint8).transpose(1, 2)[~used] = 0x7f
            b.pool[n + "s"].transpose(1, 2)[~used] = math.nan
    out, lse = run_attend(b, Q)
    assert torch.equal(out, clean) and torch.equal(lse, clean_lse)
    # a later position: only the rows from it on change
    for s, late in ((1, 47), (2, 140), (2, 165)):
        page, at = b.place(s, late)
        if form == gk.PAGES_PLAIN:
            b.pool["V"][page, :, at, 5] = math.inf
            b.pool["K"][page, :, at, 3] = math.nan
        elif form == gk.PAGES_FP8:
            b.pool["V"].view(torch.uint8)[page, :, at, 5] = 0x7f
            b.pool["Ks"][page, :, at] = math.nan
        else:
            b.pool["Vs"][page, :, at] = math.inf
            b.pool["Ks"][page, :, at] = math.nan
    out, lse = run_attend(b, Q)
    first_bad = {1: 47, 2: 140}
    for r, s, pos in b.each_row():
        if pos < first_bad.get(s, 10 ** 9):
            assert torch.equal(out[r], clean[r]) and torch.equal(lse[r], clean_lse[r]), (r, s, pos)
        else:
            assert torch.isnan(lse[r]).all() and torch.isnan(out[r]).any(), (r, s, pos)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("d,G,ps", [(64, 1, 16), (80, 3, 32), (128, 2, 64), (128, 5, 16), (96, 4, 128)])
def test_attention_of_wide_blocks(form, d, G, ps):
    """Chunks of more than 128 stacked rows (blocks of 256, tiles that pass the registers by): lengths on both sides of tiles and
    blocks, sequences that begin with the chunk, pages that are none, infinities and NaN in places that are not seen and at
    positions that some rows see."""
    say(f"wide blocks form={form} d={d} G={G} ps={ps}")
    b = pu.Batch([(150, 700), (129, 129), (3, 64), (260, 261), (64, 1025), (100, 30)], H=2, G=G, d=d, ps=ps, form=form, before=1, behind=2,
                 seed=d + G)
    b.p.max_rows = 260
    b.table[0, 2] = -1
    b.table[4, -(-1025 // ps) // 2] = b.p.n_pages
    Q = b.random_rows(2 * G, fused=4)
    clean, clean_lse = run_attend(b, Q)
    pu.check_attend(b, Q, clean, clean_lse)
    used = torch.zeros(b.p.n_pages, b.ps, dtype=torch.bool)
    for s, (_, n) in enumerate(b.pairs):
        for j in range(n):
            cell = b.place(s, j)
            if cell:
                used[cell] = True
    for n in "KV":
        if form == gk.PAGES_PLAIN:
            b.pool[n].transpose(1, 2)[~used] = math.nan
        else:
            b.pool[n].view(torch.uint8).transpose(1, 2)[~used] = 0x7f
            b.pool[n + "s"].transpose(1, 2)[~used] = math.inf
    out, lse = run_attend(b, Q)
    assert torch.equal(out, clean) and torch.equal(lse, clean_lse)
    late = {0: 640, 1: 100, 3: 200, 4: 1000}
    for s, j in late.items():
        page, at = b.place(s, j)
        if form == gk.PAGES_PLAIN:
            b.pool["V"][page, :, at, 5] = math.inf
            b.pool["V"][page, :, at, d - 1] = math.nan
        elif form == gk.PAGES_FP8:
            b.pool["V"].view(torch.uint8)[page, :, at, 5] = 0x7f
            b.pool["V"].view(torch.uint8)[page, :, at, d - 1] = 0xff
        else:
            b.pool["Vs"][page, :, at] = math.inf
    out, lse = run_attend(b, Q)
    assert torch.equal(lse, clean_lse)
    columns = [5, d - 1] if form != gk.PAGES_INT8 else list(range(d))
    rest = [c for c in range(d) if c not in columns]
    for r, s, pos in b.each_row():
        if pos < late.get(s, 10 ** 9):
            assert torch.equal(out[r], clean[r]), (r, s, pos)
        else:
            assert not torch.isfinite(out[r][:, columns]).any(), (r, s, pos)
            if rest:   # the row's other values count as before, in another order of the sum and with weights of 32 bits
                assert (out[r][:, rest].float() - clean[r][:, rest].float()).abs().max() < 0.1


def test_attention_with_large_logits_and_a_scale():
    """Logits of thousands, where only a few weights are left, and a scale of the caller's."""
    say("large logits")
    for dtype in TYPES:
        b = pu.Batch([(1, 200), (50, 190)], H=2, G=2, d=128, dtype=dtype)
        b.p.softmax_scale = 0.75
        Q = b.random_rows(4) * 8
        out, lse = run_attend(b, Q)
        pu.check_attend(b, Q, out, lse, scale=0.75)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rise", [0.03, 0.07, 0.4, -0.07])
def test_attention_with_rising_logits(dtype, rise):
    """Logits that grow, or shrink, from key to key: by less than the running reference of the softmax may stay behind from tile to
    tile, by about as much, by far more."""
    say(f"rising logits dtype={dtype} rise={rise}")
    for pairs, G, d in (([(1, 900), (3, 500)], 4, 128), ([(12, 700)], 4, 128), ([(30, 600)], 4, 64), ([(80, 500)], 4, 128)):
        b = pu.Batch(pairs, H=2, G=G, d=d, ps=32, dtype=dtype, seed=5)
        for s, (_, n) in enumerate(pairs):
            for pos in range(n):
                page, at = b.place(s, pos)
                b.pool["K"][page, :, at, 0] = rise * pos
        Q = b.random_rows(2 * G)
        Q[:, :, 0] = math.sqrt(d)
        out, lse = run_attend(b, Q)
        pu.check_attend(b, Q, out, lse)


@pytest.mark.parametrize("d", [64, 80, 128, 256])
def test_attention_of_few_rows_keeps_the_weights(d):
    """At most 32 stacked rows over plain pages in bf16: the weights go into the product with the values as two bf16 numbers each, the first
    cut off, the second rounded: what the first leaves is at most 2^-7 of the weight, and half a step of that 2^-8 of it, so a weight is off by
    2^-15 (and by the 2^-22 that the second is made larger by), not by 2^-8."""
    say(f"weights of few rows d={d}")
    b = pu.Batch([(1, 2), (1, 3), (1, 40), (2, 300), (8, 100), (3, 2), (1, 2000)], H=2, G=4, d=d, ps=16, before=1, behind=1, seed=d)
    Q = b.random_rows(8)
    out, lse = run_attend(b, Q)
    pu.check_attend(b, Q, out, lse)
    want, _, bound, _ = b.attend(Q)
    values, b.pool["V"] = b.pool["V"], b.pool["V"].abs()
    mass = b.attend(Q)[0]   # sums of the magnitudes
    b.pool["V"] = values
    mine = ~want.isnan()
    allow = bound - (2.0 ** -8 - 2.0 ** -15 - 2.0 ** -22) * mass
    assert ((out.cpu().double() - want).abs() <= allow + 2.0 ** -100)[mine].all()


# (stacked rows: 32, 8, 48, 120, 320; which kernel takes them goes by the type of the rows and d too)
OTHERS = [([(8, 500)], 4, 128), ([(4, 300)], 2, 64), ([(12, 700)], 4, 128), ([(30, 600)], 4, 64), ([(30, 600)], 4, 128), ([(80, 500)], 4, 128),
          ([(80, 500)], 4, 64), ([(40, 300)], 1, 256)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("shape", range(len(OTHERS)))
def test_attention_does_not_depend_on_other_rows(dtype, form, shape):
    """Logits that grow a little from key to key, so that the running reference of a softmax may stay behind: a large finite key at a late
    position, or other queries of the later rows, leave the earlier rows' bits as they are."""
    pairs, G, d = OTHERS[shape]
    say(f"other rows dtype={dtype} form={form} {pairs} G={G} d={d}")
    (n, length), = pairs
    for rise in (0.004, 0.012, 0.03):
        b = pu.Batch(pairs + [(1, 32)], H=2, G=G, d=d, ps=32, dtype=dtype, form=form, seed=shape, table_pages=4096)
        b.len[1] = 4096 * 32   # (beside a long sequence a workgroup's stretch holds several tiles of the first one)
        keys = torch.randn(b.p.n_pages, 2, 32, d, generator=b.g)
        for pos in range(length):
            page, at = b.place(0, pos)
            keys[page, :, at, 0] = rise * pos
        b.set_pool("K", keys.to(b.p.torch_dtype))
        Q = b.random_rows(2 * G)
        Q[:, :, 0] = math.sqrt(d)
        clean, clean_lse = run_attend(b, Q)
        if rise == 0.03:
            pu.check_attend(b, Q, clean, clean_lse)
        for late in (length - n + n // 2, length - 2):
            before = late - (length - n)   # rows of the sequence that do not see the late position
            page, at = b.place(0, late)
            own_key = keys[page, :, at].clone()
            for value in (60.0, 3000.0, math.inf) if form == gk.PAGES_PLAIN else (60.0, 3000.0):
                keys[page, :, at] = 0
                keys[page, :, at, 0] = value
                b.set_pool("K", keys.to(b.p.torch_dtype))
                out, lse = run_attend(b, Q)
                assert torch.equal(out[:before], clean[:before]) and torch.equal(lse[:before], clean_lse[:before]), (rise, late, value)
                assert not torch.equal(lse[before:n], clean_lse[before:n])
            keys[page, :, at] = own_key
            b.set_pool("K", keys.to(b.p.torch_dtype))
            other = Q.clone()
            other[before:n] *= 7
            out, lse = run_attend(b, other)
            assert torch.equal(out[:before], clean[:before]) and torch.equal(lse[:before], clean_lse[:before]), (rise, late)


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_of_many_sequences(dtype):
    """More sequences than a workgroup has threads, most of them short, some without new rows."""
    say(f"many sequences dtype={dtype}")
    g = torch.Generator().manual_seed(11)
    pairs = [(int(torch.randint(0, 3, (1,), generator=g)), int(torch.randint(2, 40, (1,), generator=g))) for _ in range(300)]
    pairs[290] = (40, 60)
    b = pu.Batch(pairs, H=1, G=2, d=64, ps=8, dtype=dtype, before=1, behind=1)
    Q = b.random_rows(2)
    out, lse = run_attend(b, Q)
    pu.check_attend(b, Q, out, lse)


LONG = [([(1, 9001)], 1, 4, 128), ([(8, 20000), (1, 30)], 1, 4, 128), ([(1, 70000), (1, 9)], 2, 1, 64), ([(1, 12000)], 1, 2, 256), ([(12, 9000)], 1, 4, 128),
        ([(30, 10001)], 1, 4, 128), ([(100, 6000)], 1, 1, 64), ([(60, 12000), (5, 3000)], 1, 4, 128), ([(300, 4100)], 2, 1, 64), ([(40, 5000)], 1, 4, 256),
        ([(1, 4000)] * 8 + [(200, 7000)], 1, 2, 128)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("shape", range(len(LONG)))
def test_attention_over_many_parts(dtype, form, shape):
    """Long sequences of few heads, whose keys are shared out among many workgroups and joined from as many parts, against the definition."""
    pairs, H, G, d = LONG[shape]
    say(f"many parts dtype={dtype} form={form} {LONG[shape]}")
    b = pu.Batch(pairs, H=H, G=G, d=d, ps=64, dtype=dtype, form=form, seed=shape, before=1, behind=1)
    Q = b.random_rows(H * G)
    out, lse = run_attend(b, Q)
    out, lse = out.cpu().double(), lse.cpu().double()
    k, v, c, u = b.values("K"), b.values("V"), 1 / math.sqrt(d), 2.0 ** -24
    for s, (n, length) in enumerate(pairs):
        pages = b.table[s, :-(-length // 64)].long()
        r0 = int(b.start[s])
        hidden = torch.arange(length)[None] > torch.arange(length - n, length)[:, None]
        for h in range(H * G):
            kk, vv = (x[pages, h // G].reshape(-1, d)[:length] for x in (k, v))
            q = Q[r0:r0 + n, h].double()
            x = (q @ kk.T * c).masked_fill(hidden, -math.inf)
            w = torch.softmax(x, 1)
            want, want_lse = w @ vv, torch.logsumexp(x, 1)
            # as the tests of short sequences: logits, sums, weights and results, each with its rounding
            off = (d + 8) * u * (q.abs() @ kk.abs().T).amax(1) * c
            terms = (length + d + 64) * u
            weights = pu.half_step(torch.bfloat16) if dtype == gk.BF16 else 0.0
            bound = (w @ vv.abs()) * (weights + 4 * off + 4 * terms)[:, None] + want.abs() * pu.half_step(b.p.torch_dtype)
            assert ((out[r0:r0 + n, h] - want).abs() <= bound).all(), (s, h)
            assert ((lse[r0:r0 + n, h] - want_lse).abs() <= 2 * off + 2 * terms + want_lse.abs() * 8 * u).all(), (s, h)


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_over_the_longest_tables(dtype):
    """Tables of 2^30 tokens with more heads and sequences than the kernel for few rows would count, which takes none of them."""
    say(f"longest tables dtype={dtype}")
    b = pu.Batch([(40, 100), (40, 1500), (33, 33), (1, 0)], H=64, G=1, d=16, ps=1024, dtype=dtype, table_pages=1 << 20, behind=1)
    assert b.p.table_pages * b.ps == 1 << 30 and 4 * 64 * (1 << 30) // 128 >= 1 << 31
    Q = b.random_rows(64)
    out, lse = run_attend(b, Q)
    pu.check_attend(b, Q, out, lse)


# ---- together, in graphs, on streams ----------------------------------------------------------------

def test_prefill_evict_decode():
    """The calls as a serving loop makes them: chunks of a prompt written and attended over, the prompt read back and evicted, what
    is kept written to fewer pages, tokens generated behind it."""
    say("prefill, evict, decode")
    H, G, d, ps, N, w, B = 2, 4, 128, 32, 700, 16, 150
    g = torch.Generator("cuda").manual_seed(3)
    for form in FORMS:
        pool = [torch.zeros(40, H, ps, d, device="cuda").to(pu.CODE.get(form, torch.bfloat16)) for _ in range(2)]
        scales = [] if form == gk.PAGES_PLAIN else [torch.zeros(40, H, ps, device="cuda") for _ in range(2)]
        qkv = torch.randn(N, (G + 2) * H, d, generator=g, device="cuda").to(torch.bfloat16)
        Q, K, V = qkv[:, :G * H], qkv[:, G * H:G * H + H], qkv[:, G * H + H:]
        table = torch.randperm(40, generator=g, device="cuda").to(torch.int32)[None, :24].contiguous()
        p = gk.PagedParams(n_kv_heads=H, n_q_heads=G * H, head_dim=d, page_tokens=ps, n_pages=40, n_seqs=1, table_pages=24, n_rows=0,
                           page_format=form)
        i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
        out = torch.empty(N, G * H, d, dtype=torch.bfloat16, device="cuda")
        for a, e in ((0, 1), (1, 300), (300, 311), (311, N)):
            p.n_rows = e - a
            batch = (table, i32(e), i32(0, e - a))
            gk.graphkv_cache_write(p, K[a:e], V[a:e], *pool, *batch, *scales)
            gk.graphkv_attend(p, Q[a:e], *pool, *batch, *scales, out=out[a:e])
        # the whole prompt again as one batch of rows, [H, N, d] as the eviction pass takes it
        p.n_rows = N
        batch = (table, i32(N), i32(0, N))
        Kc, Vc = (torch.empty(H, N, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        gk.graphkv_cache_read(p, *pool, *batch, *scales, K=Kc.transpose(0, 1), V=Vc.transpose(0, 1))
        if form == gk.PAGES_PLAIN:
            assert torch.equal(Kc, K.transpose(0, 1)) and torch.equal(Vc, V.transpose(0, 1))
        hidden = torch.ones(N, N, dtype=torch.bool, device="cuda").triu(1)
        k, v = (t.double().repeat_interleave(G, 0) for t in (Kc, Vc))
        x = (Q.transpose(0, 1).double().contiguous() @ k.transpose(1, 2).contiguous() / math.sqrt(d)).masked_fill(hidden, -math.inf)
        want = (torch.softmax(x, -1) @ v).transpose(0, 1)
        # weights of bf16, and for coded pages values that were rounded to bf16 on their way back, as the keys were
        allow = 2 * pu.half_step(torch.bfloat16) * (torch.softmax(x, -1) @ v.abs()).transpose(0, 1) + pu.half_step(torch.bfloat16) * want.abs()
        if form != gk.PAGES_PLAIN:
            shift = pu.half_step(torch.bfloat16) * (Q.transpose(0, 1).double().abs().contiguous() @ k.abs().transpose(1, 2).contiguous()).amax(-1) / math.sqrt(d)
            allow = allow + (2 * shift.T[..., None] + pu.half_step(torch.bfloat16)) * (torch.softmax(x, -1) @ v.abs()).transpose(0, 1)
        assert ((out.double() - want).abs() <= allow + 1e-4).all()
        # eviction, the kept rows to five other pages
        ep = gk.Params(n_kv_heads=H, n_q_heads=G * H, head_dim=d, n_tokens=N, window=w, pool_kernel=5, budget=B, n_sources=8, n_neighbors=4, rounds=1)
        Ko, Vo, idx = gk.graphkv_compress(ep, Kc, Vc, Q[N - w:].transpose(0, 1).contiguous())
        kept = torch.arange(30, 35, device="cuda", dtype=torch.int32)[None].contiguous()
        kp = gk.PagedParams(n_kv_heads=H, n_q_heads=G * H, head_dim=d, page_tokens=ps, n_pages=40, n_seqs=1, table_pages=5, n_rows=B, page_format=form)
        gk.graphkv_cache_write(kp, Ko.transpose(0, 1), Vo.transpose(0, 1), *pool, kept, i32(B), i32(0, B), *scales)
        kp.n_rows = 1
        for step in range(3):
            new = torch.randn(1, (G + 2) * H, d, generator=g, device="cuda").to(torch.bfloat16)
            batch = (kept, i32(B + 1 + step), i32(0, 1))
            gk.graphkv_cache_write(kp, new[:, G * H:G * H + H], new[:, G * H + H:], *pool, *batch, *scales)
            got = gk.graphkv_attend(kp, new[:, :G * H], *pool, *batch, *scales)
            b = pu.Batch([(1, B + 1 + step)], H=H, G=G, d=d, ps=ps, form=form)
            b.p, b.table = kp, kept.cpu()
            b.pool = {n: t.cpu() for n, t in zip(("K", "V", "Ks", "Vs"), pool + scales)}
            pu.check_attend(b, new[:, :G * H].cpu(), got)


@pytest.mark.parametrize("pairs,d,form", [([(1, 60)] * 3 + [(1, 900)], 128, gk.PAGES_PLAIN), ([(8, 200), (1, 40), (100, 150)], 128, gk.PAGES_FP8),
                                          ([(40, 90)], 64, gk.PAGES_INT8)])
def test_captured_calls_follow_the_lengths(pairs, d, form):
    """A captured write and attention, replayed with other rows, lengths and pages, with eager work between: the eager calls' bits."""
    say(f"captured calls {pairs} d={d} form={form}")
    b = pu.Batch(pairs, H=2, G=4, d=d, ps=16, form=form, behind=3, table_pages=80, spare=80 * len(pairs))
    # (every page once, whatever the lengths: no two rows of a write may have the same place)
    b.table = torch.randperm(b.p.n_pages, generator=b.g)[:80 * len(pairs)].reshape(-1, 80).int()
    K, V, Q = (on_gpu(b.random_rows(h)) for h in (2, 2, 8))
    args = b.device()
    ws = gk.alloc_attend_workspace(b.p)
    out, lse = torch.zeros(b.rows, 8, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(b.rows, 8, device="cuda")

    def step(o, le, w):
        gk.graphkv_cache_write(b.p, K, V, *args)
        gk.graphkv_attend(b.p, Q, *args, out=o, lse=le, ws=w)

    step(out, lse, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, lse, ws)
    g = torch.Generator("cuda").manual_seed(1)
    for n in range(4):
        for t in (K, V, Q):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        lens = torch.tensor([min(m + 37 * n, 1200) for _, m in pairs], dtype=torch.int32)
        if n == 2:
            lens[0] = 0
        args[3].copy_(lens)
        args[2].copy_(args[2].roll(n, 1))
        pools = [t.clone() for t in args[:2] + args[5:]]
        graph.replay()
        torch.cuda.synchronize()
        got, got_lse, got_pools = out.clone(), lse.clone(), [t.clone() for t in args[:2] + args[5:]]
        for t, was in zip(args[:2] + args[5:], pools):
            t.copy_(was)
        want, want_lse = torch.zeros_like(out), torch.zeros_like(lse)
        step(want, want_lse, torch.randint(0, 256, ws.shape, dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(got_lse, want_lse), f"replay {n}"
        for x, y in zip(got_pools, args[:2] + args[5:]):
            assert torch.equal(bits(x), bits(y))


def test_graphs_that_share_a_workspace():
    """Captured calls of either kernel, of both and of blocks of each size leave nothing in the workspace that the next one would
    take for its own: replayed in turn, with eager calls on the same workspace between."""
    say("graphs that share a workspace")
    sets = []
    for seed, pairs in ((1, [(1, 3000), (1, 5), (1, 900)]), (2, [(60, 500), (1, 700)]), (3, [(1, 300)] * 9 + [(70, 400), (4, 90)]), (4, [(14, 800)])):
        b = pu.Batch(pairs, H=2, G=4, d=128, ps=16, seed=seed)
        sets.append((b, on_gpu(b.random_rows(8)), b.device()))
    ws = torch.randint(0, 256, (max(gk.graphkv_attend_workspace_bytes(b.p) for b, _, _ in sets),), dtype=torch.uint8, device="cuda")
    want = [gk.graphkv_attend(b.p, Q, *args) for b, Q, args in sets]
    torch.cuda.synchronize()
    graphs = []
    for b, Q, args in sets:
        out, graph = torch.zeros_like(Q), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            gk.graphkv_attend(b.p, Q, *args, out=out, ws=ws)
        graphs.append((graph, out))
    for turn in ([0, 1, 2, 3], [3, 2, 1, 0], [2, 2, 0, 3, 1]):
        for i in turn:
            graphs[i][1].zero_()
            graphs[i][0].replay()
            b, Q, args = sets[(i + 1) % len(sets)]
            assert torch.equal(gk.graphkv_attend(b.p, Q, *args, ws=ws), want[(i + 1) % len(sets)])
        torch.cuda.synchronize()
        for i in turn:
            assert torch.equal(graphs[i][1], want[i]), (turn, i)


def test_two_streams_with_a_workspace_each():
    say("two streams")
    sets = []
    for seed, pairs in ((1, [(1, 3000)]), (2, [(60, 500), (1, 700)])):
        b = pu.Batch(pairs, H=2, G=4, d=128, ps=16, seed=seed)
        Q = on_gpu(b.random_rows(8))
        args = b.device()
        sets.append((b, Q, args, gk.alloc_attend_workspace(b.p), gk.graphkv_attend(b.p, Q, *args), torch.cuda.Stream()))
    torch.cuda.synchronize()
    outs = []
    for _ in range(5):
        for b, Q, args, ws, want, stream in sets:
            with torch.cuda.stream(stream):
                outs.append((gk.graphkv_attend(b.p, Q, *args, ws=ws), want))
    torch.cuda.synchronize()
    for got, want in outs:
        assert torch.equal(got, want)


def test_strided_outputs_leave_the_rest_alone():
    say("strided outputs")
    b = pu.Batch([(3, 40), (50, 90)], H=2, G=2, d=64, ps=16)
    Q, args = on_gpu(b.random_rows(4)), b.device()
    want = gk.graphkv_attend(b.p, Q, *args)
    wide = torch.full((b.rows, 6, 96), -7.0, dtype=torch.bfloat16, device="cuda")
    gk.graphkv_attend(b.p, Q, *args, out=wide[:, 1:5, 16:80])
    assert torch.equal(wide[:, 1:5, 16:80], want)
    wide[:, 1:5, 16:80] = -7
    assert (wide == -7).all()
    by_head = torch.empty(4, b.rows, 64, dtype=torch.bfloat16, device="cuda")
    gk.graphkv_attend(b.p, Q, *args, out=by_head.transpose(0, 1))
    assert torch.equal(by_head.transpose(0, 1), want)


def test_binding_refuses_wrong_tensors():
    say("wrong tensors")
    b = pu.Batch([(3, 40)], H=2, G=2, d=64, ps=16, form=gk.PAGES_INT8)
    Q, args = on_gpu(b.random_rows(4)), b.device()
    K = on_gpu(b.random_rows(2))
    good = lambda: list(args)

    def refuse(match, f, *a, **kw):
        with pytest.raises(gk.GraphKVError, match=match):
            f(b.p, *a, **kw)

    for i, bad in ((0, args[0].to(torch.uint8)), (0, args[0][:-1]), (1, args[1].transpose(0, 1)), (2, args[2].long()), (3, args[3][:0]),
                   (4, args[4].cpu()), (5, args[5].double()), (6, None)):
        a = good()
        a[i] = bad
        refuse(".", gk.graphkv_attend, Q, *a)
    refuse("shape", gk.graphkv_attend, Q[:-1], *args)
    refuse("dtype", gk.graphkv_attend, Q.float(), *args)
    refuse("strides", gk.graphkv_attend, Q.expand(3, 4, 64)[:1].expand(3, 4, 64), *args)
    refuse("strides", gk.graphkv_attend, torch.empty(3, 4, 128, dtype=torch.bfloat16, device="cuda")[..., ::2], *args)
    refuse("same strides", gk.graphkv_cache_write, K, on_gpu(b.random_rows(2, by_head=True)), *args)
    refuse("lse", gk.graphkv_attend, Q, *args, lse=torch.empty(3, 3, device="cuda"))
    refuse("-2", gk.graphkv_attend, Q, *args, ws=torch.empty(16, dtype=torch.uint8, device="cuda"))
    refuse("-1", gk.graphkv_attend, Q, *args, out=torch.empty(400, dtype=torch.bfloat16, device="cuda").as_strided((3, 4, 64), (64, 64, 1)))
    torch.cuda.synchronize()
