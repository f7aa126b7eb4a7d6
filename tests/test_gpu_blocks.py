"""Pages of 8-bit codes with a scale for each block of tokens and head: written, read back, attended over, against their
definitions in 64 bits (GPU)."""
import math

import pytest
import torch

from paper_2509_00388_amd import binding as gk
from tests import more_util as mu
from tests import paged_util as pu
from tests.test_gpu_paged import LONG, OTHERS, bits, on_gpu, run_attend, say

pytestmark = pytest.mark.gpu

TYPES = [gk.BF16, gk.FP32]
IMPLS = [gk.IMPL_AUTO, gk.IMPL_GENERIC]


# ---- write and read ---------------------------------------------------------------------------------

def check_write(b, K, V, args=None):
    want = mu.written(b, K, V)
    args = args or b.device()
    gk.graphkv_cache_write(b.p, on_gpu(K), on_gpu(V), *args)
    for n, got in zip(("K", "V", "Ks", "Vs"), args[:2] + args[5:]):
        assert torch.equal(bits(got), bits(want[n])), f"pool {n}"
    b.pool = want
    return args


def check_read(b, args, by_head=False):
    shape = (b.H, b.rows, b.d) if by_head else (b.rows, b.H, b.d)
    K, V = (torch.full(shape, -7.0, dtype=b.p.torch_dtype, device="cuda") for _ in range(2))
    if by_head:
        K, V = K.transpose(0, 1), V.transpose(0, 1)
    gk.graphkv_cache_read(b.p, *args, K=K, V=V)
    for n, got in (("K", K), ("V", V)):
        want = torch.full((b.rows, b.H, b.d), -7.0, dtype=torch.float64)
        values = b.values(n)
        for r, s, pos in b.each_row():
            cell = b.place(s, pos)
            want[r] = 0.0 if cell is None else values[cell[0], :, cell[1]]
        # (the product in 64 bits is exact, so this rounds once)
        assert torch.equal(got.cpu(), want.to(b.p.torch_dtype))


def spread(b, H, **kw):
    """Rows whose sizes differ from token to token and head to head."""
    x = b.random_rows(H, **kw)
    x *= torch.exp(2 * torch.randn(b.rows, H, 1, generator=b.g)).to(x.dtype)
    return x


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", mu.BLOCKS)
@pytest.mark.parametrize("d,H,ps,block,how", [(64, 2, 16, 16, "packed"), (128, 8, 64, 32, "fused"), (80, 3, 32, 16, "by_head"), (16, 5, 128, 128, "packed"),
                                              (512, 1, 64, 16, "fused"), (256, 7, 32, 32, "by_head"), (128, 2, 512, 256, "packed")])
def test_rows_written_and_read_back(dtype, form, d, H, ps, block, how):
    """Blocks that begin, end and lie within a call's rows; blocks that hold tokens already, sequences without new rows."""
    say(f"write and read blocks dtype={dtype} form={form} d={d} H={H} ps={ps} block={block} {how}")
    b = mu.Batch([(1, 1), (5, 40), (0, 17), (33, 33), (7, 130), (300, 700), (1, 513)], form=form, block=block, H=H, d=d, ps=ps, dtype=dtype,
                 before=2, behind=3, seed=d + H)
    kw = dict(by_head=how == "by_head", fused=4 if how == "fused" else 0)
    args = check_write(b, spread(b, H, **kw), spread(b, H, **kw))
    check_read(b, args, by_head=how != "packed")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", mu.BLOCKS)
def test_blocks_grow_token_by_token(dtype, form):
    """Tokens appended one and a few at a time, each larger or smaller than those before: every state by the definition, and values never
    further off than the scales they went through allow."""
    say(f"blocks grow dtype={dtype} form={form}")
    H, d, ps, block = 3, 64, 32, 16
    g = torch.Generator().manual_seed(int(form))
    n = 70
    rows = (torch.randn(2, n, H, d, generator=g) * torch.exp(1.5 * torch.randn(2, n, H, 1, generator=g))).to(pu.TORCH[dtype])
    rows[:, 20:24] = 0                                   # rows of zeros
    rows[:, 32:36] = 0                                   # a block that begins with them
    rows[:, 40] *= 1e4
    rows[:, 48:50] *= 2.0 ** -110                        # next to nothing
    b = mu.Batch([(1, n)], form=form, block=block, H=H, d=d, ps=ps, dtype=dtype, spare=1)
    args, at = None, 0
    for step in [1] * 20 + [3, 1, 2, 7, 5, 1, 1, 1, 9, 17, 1, 1, 1]:
        b.p.n_rows = b.p.max_rows = b.rows = step
        b.len, b.start = torch.tensor([at + step], dtype=torch.int32), torch.tensor([0, step], dtype=torch.int32)
        if args:
            args[3], args[4] = b.len.cuda(), b.start.cuda()
        args = check_write(b, rows[0, at:at + step], rows[1, at:at + step], args)
        at += step
    assert at == n
    table = b.table[0].long()
    for i, name in enumerate("KV"):
        got = b.values(name)[table].transpose(1, 2).reshape(-1, H, d)[:n]
        scale = b.pool[name + "s"].double()[table].transpose(1, 2).reshape(-1, H).repeat_interleave(block, 0)[:n]
        # a code is off by half a step of its scale, once for each time that its block's scale grew: integers by 1/2 of it
        # each, the scales growing to this one; e4m3 by 2^-4 of the value each, or by half of its least step, 2^-10
        x = rows[i].double()
        if form == gk.PAGES_INT8_BLOCKS:
            # a token's code is rounded again at most once for each later token of its block
            later = (block - 1 - torch.arange(n) % block).double()[:, None]
            allow = (0.5 * (1 + later) * scale)[..., None].expand_as(x)
        else:
            # scales double at least when they grow, and codes of 2^-6 and more keep their bits: only the first rounding and those below count
            allow = x.abs() * 2.0 ** -4 + (2 * 2.0 ** -10 * scale)[..., None]
        assert ((got - x).abs() <= allow * (1 + 1e-6) + 2.0 ** -100).all()


def test_rows_without_a_place():
    """Negative positions, page numbers that are none, rows of no sequence: nothing else changes."""
    say("rows without a place")
    for form in mu.BLOCKS:
        b = mu.Batch([(50, 20), (4, 60), (6, 90), (3, 0), (40, 70)], form=form, block=16, H=2, d=64, ps=32, before=2, behind=2, spare=4)
        b.table[1, 1], b.table[2, 2], b.table[4, 1] = -1, b.p.n_pages, 2 ** 31 - 1
        args = check_write(b, spread(b, 2), spread(b, 2))
        check_read(b, args)


@pytest.mark.parametrize("dtype", TYPES)
def test_many_sequences_and_rows(dtype):
    """More rows than are looked at one by one, in sequences longer and shorter than a block."""
    say(f"many sequences dtype={dtype}")
    g = torch.Generator().manual_seed(2)
    for pairs, block in (([(1, int(n)) for n in torch.randint(1, 200, (700,), generator=g)], 32), ([(2900, 3000), (40, 41), (1, 5), (700, 700)], 16),
                         ([(int(n) % 40, int(n)) for n in torch.randint(0, 200, (150,), generator=g)], 16)):
        b = mu.Batch(pairs, form=gk.PAGES_FP8_BLOCKS, block=block, H=8, d=16, ps=64, dtype=dtype, before=1, behind=1)
        check_write(b, spread(b, 8), spread(b, 8))


def test_as_many_blocks_as_rows_can_lie_in():
    """Rows that begin with a block's last token and end with one's first; calls that do not tell how many rows a sequence has."""
    say("as many blocks as rows can lie in")
    for n, seqs in ((1, 130), (2, 130), (18, 100), (34, 65), (18, 1), (2, 1)):
        for max_rows in (n, n * seqs):
            b = mu.Batch([(n, 15 + n + 16 * (s % 3)) for s in range(seqs)], form=gk.PAGES_INT8_BLOCKS, block=16, H=5, d=64, ps=32, max_rows=max_rows)
            check_write(b, spread(b, 5), spread(b, 5))


@pytest.mark.parametrize("form", mu.BLOCKS)
def test_writes_with_numbers_of_any_content(form):
    """Lengths, row numbers and page numbers without any sense: nothing around the pools is touched."""
    say(f"writes with numbers of any content form={form}")
    g = torch.Generator().manual_seed(17)
    H, d, ps, pages, block = 3, 64, 32, 40, 16
    pool = pages * H * ps * d
    for n_seqs, rows in ((1, 9), (70, 300), (200, 1)):
        p = gk.PagedParams(n_kv_heads=H, head_dim=d, page_tokens=ps, n_pages=pages, n_seqs=n_seqs, table_pages=6, n_rows=rows, page_format=form,
                           scale_tokens=block)
        x = torch.randn(rows, H, d, generator=g).to(torch.bfloat16).cuda()
        for kind in range(4):
            codes = [torch.full((pool + 512,), 77, dtype=torch.uint8, device="cuda") for _ in range(2)]
            scales = [torch.full((pages * H * ps // block + 128,), 77.0, device="cuda") for _ in range(2)]
            big = [3, 2 ** 31 - 1, 2 ** 10, 2 ** 20][kind]
            numbers = [torch.randint(-big, big, shape, generator=g).int().cuda() for shape in ((n_seqs, 6), (n_seqs,), (n_seqs + 1,))]
            table, length, start = numbers
            if kind == 2:
                table = torch.randint(0, pages, (n_seqs, 6), generator=g).int().cuda()
            t = torch.int8 if form == gk.PAGES_INT8_BLOCKS else torch.float8_e4m3fn
            K, V = (c[256:-256].view(t).view(pages, H, ps, d) for c in codes)
            Ks, Vs = (c[64:-64].view(pages, H, ps // block) for c in scales)
            gk.graphkv_cache_write(p, x, x, K, V, table, length, start, Ks, Vs)
            for c in codes:
                assert (c[:256] == 77).all() and (c[-256:] == 77).all()
            for c in scales:
                assert (c[:64] == 77).all() and (c[-64:] == 77).all()


def test_codes_next_to_borders():
    """Values in the middle between two codes and one step of their type next to it, new ones and ones that are rounded again."""
    say("codes next to borders")
    for dtype in TYPES:
        t = pu.TORCH[dtype]
        for form in mu.BLOCKS:
            b = mu.Batch([(2, 2)], form=form, block=16, H=1, d=128, ps=16, dtype=dtype, spare=0)
            top = 448.0 if form == gk.PAGES_FP8_BLOCKS else 127.0
            every = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).float() if form == gk.PAGES_FP8_BLOCKS else torch.arange(127.0)
            mid = ((every[1:] + every[:-1]) / 2).to(t)      # (five bits, or eight)
            K = torch.zeros(2, 1, 128, dtype=t)
            K[0, 0, 0], K[1, 0, 0] = top, 3.0
            K[0, 0, 1:127] = mid
            K[1, 0, 1:127] = torch.nextafter(mid, torch.full_like(mid, 1e9))
            V = -K
            args = check_write(b, K, V)
            for factor in (2.0, 3.0, 1.7):       # a third token of another size: the codes above are rounded again
                b.p.n_rows = b.p.max_rows = b.rows = 1
                b.len, b.start = b.len + 1, torch.tensor([0, 1], dtype=torch.int32)
                args[3], args[4] = b.len.cuda(), b.start.cuda()
                x = torch.zeros(1, 1, 128, dtype=t)
                x[0, 0, 5] = float(b.pool["Ks"]) * top * factor
                args = check_write(b, x, -x, args)


# ---- attention --------------------------------------------------------------------------------------

SHAPES = [
    dict(pairs=[(1, 1)], H=1, G=1, d=128), dict(pairs=[(1, 129), (1, 31), (1, 1), (1, 512)], H=2, G=4, d=128, ps=64, block=32),
    dict(pairs=[(1, 700), (1, 64)], H=3, G=7, d=64, ps=32), dict(pairs=[(1, 300)] * 5, H=2, G=32, d=80, ps=128, block=128),
    dict(pairs=[(8, 100), (3, 3), (1, 250)], H=2, G=4, d=128, ps=64, block=64), dict(pairs=[(4, 77)], H=1, G=8, d=64, ps=16),
    dict(pairs=[(100, 300)], H=2, G=4, d=128), dict(pairs=[(33, 33)], H=3, G=1, d=64, ps=32, block=32),
    dict(pairs=[(1, 150), (70, 200), (8, 90), (129, 130)], H=2, G=2, d=128, ps=32),
    dict(pairs=[(19, 260), (0, 50), (50, 50)], H=2, G=7, d=96, ps=128, block=64),
    dict(pairs=[(1, 150), (70, 200), (8, 90), (129, 130), (1, 1), (1, 33), (2, 64), (0, 9), (1, 400)], H=2, G=2, d=128, ps=32, block=32),
    dict(pairs=[(1, 90), (30, 60), (2, 90), (1, 0), (1, 7), (1, 33), (5, 64), (3, 2), (40, 100)], H=2, G=7, d=64, ps=16),
    dict(pairs=[(150, 700), (129, 129), (3, 64), (260, 261), (64, 1025), (100, 30)], H=1, G=2, d=128, ps=64, block=32),
    dict(pairs=[(150, 700), (260, 261)], H=2, G=1, d=64, ps=16), dict(pairs=[(200, 330)], H=1, G=2, d=112, ps=256, block=256),
    dict(pairs=[(1, 200), (40, 140)], H=2, G=2, d=256, block=16), dict(pairs=[(3, 120)], H=2, G=2, d=160, ps=64, block=32),
    dict(pairs=[(2, 90), (20, 60)], H=1, G=2, d=512), dict(pairs=[(1, 100), (45, 45)], H=2, G=1, d=16), dict(pairs=[(1, 140)], H=1, G=48, d=64),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", mu.BLOCKS)
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_attention(dtype, form, shape):
    say(f"attention over blocks dtype={dtype} form={form} {SHAPES[shape]}")
    b = mu.Batch(dtype=dtype, form=form, before=1, behind=2, seed=shape, **SHAPES[shape])
    Q = b.random_rows(b.H * b.G, fused=2 * b.H)
    out, lse = run_attend(b, Q)
    pu.check_attend(b, Q, out, lse)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", mu.BLOCKS)
def test_attention_scalar_kernel(dtype, form):
    say(f"attention over blocks, scalar kernel dtype={dtype} form={form}")
    b = mu.Batch([(1, 400), (30, 300), (4, 2)], H=2, G=2, d=80, ps=32, block=32, dtype=dtype, form=form, impl=gk.IMPL_GENERIC, before=1, behind=1)
    assert gk.graphkv_attend_workspace_bytes(b.p) == 0
    Q = b.random_rows(4)
    out, lse = run_attend(b, Q)
    pu.check_attend(b, Q, out, lse)


@pytest.mark.parametrize("impl", IMPLS)
@pytest.mark.parametrize("form", mu.BLOCKS)
@pytest.mark.parametrize("pairs", [[(1, 300), (3, 90)], [(60, 300), (40, 90)]])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_of_large_and_small_numbers(form, impl, pairs, d):
    """Queries and keys of 32 bits far from 1, whose products are not; values of all sizes."""
    say(f"large and small numbers form={form} impl={impl} {pairs} d={d}")
    for query, key, value, scale in ((100, -70, 90, -30), (-60, 60, -60, 0), (0, -95, 0, 95), (40, 40, 60, -80)):
        b = mu.Batch(pairs, H=2, G=2, d=d, ps=32, block=16, dtype=gk.FP32, form=form, impl=impl, before=1, behind=1, seed=query + 100)
        for n, e in (("K", key), ("V", value)):
            x = b.values(n)
            b.set_pool(n, (x / x.abs().max() * 2.0 ** e * 3).float())
        Q = b.random_rows(4) * 2.0 ** query
        b.p.softmax_scale = 2.0 ** scale / math.sqrt(d)
        out, lse = run_attend(b, Q)
        pu.check_attend(b, Q, out, lse, scale=2.0 ** scale / math.sqrt(d))


@pytest.mark.parametrize("impl", IMPLS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", mu.BLOCKS)
@pytest.mark.parametrize("pairs", [[(1, 300), (3, 90)], [(60, 300), (40, 90)]])
def test_attention_of_queries_that_are_no_numbers(dtype, form, impl, pairs):
    """Infinities of both signs and NaN of any bits in a query: NaN in its output, the others' bits as without."""
    say(f"queries that are no numbers dtype={dtype} form={form} impl={impl} {pairs}")
    b = mu.Batch(pairs, H=2, G=2, d=128, ps=32, block=16, dtype=dtype, form=form, impl=impl)
    Q = b.random_rows(4)
    want, want_lse = run_attend(b, Q)
    odd = [math.inf, -math.inf, math.nan]
    if dtype == gk.FP32:
        odd.append(torch.tensor([0x7f800001], dtype=torch.int32).view(torch.float32))   # (all but the last of its bits are an infinity's)
    for i, x in enumerate(odd):
        for r, h, c in ((0, 1, 5), (b.rows - 1, 3, 127), (2, 0, 0)):
            T = Q.clone()
            T[r, h, c] = x
            out, lse = run_attend(b, T)
            assert out[r, h].isnan().all() and lse[r, h].isnan()
            rest = torch.ones(b.rows, 4, dtype=torch.bool)
            rest[r, h] = False
            assert torch.equal(bits(out.cpu()[rest]), bits(want.cpu()[rest])) and torch.equal(bits(lse.cpu()[rest]), bits(want_lse.cpu()[rest]))


@pytest.mark.parametrize("impl", IMPLS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", mu.BLOCKS)
def test_attention_over_blocks_without_a_scale(dtype, form, impl):
    """Blocks of zeros have scale 0: their keys' logits are 0 and their values add nothing; small and large scales side by side; pages that are none."""
    say(f"blocks without a scale dtype={dtype} form={form} impl={impl}")
    for pairs in ([(1, 300), (3, 90), (2, 16)], [(60, 300), (40, 90)], [(200, 300), (20, 40)]):
        b = mu.Batch(pairs, H=2, G=2, d=64, ps=32, block=16, dtype=dtype, form=form, impl=impl, before=1, behind=1, spare=3)
        for n in "KV":
            x = b.values(n).reshape(b.p.n_pages, 2, 2, 16, 64)
            size = torch.exp2(torch.randint(-9, 4, (b.p.n_pages, 2, 2, 1, 1), generator=b.g).double())
            size[torch.rand(size.shape, generator=b.g) < 0.3] = 0
            b.set_pool(n, (x * size).reshape(b.p.n_pages, 2, 32, 64).to(b.p.torch_dtype))
        b.table[0, 3] = -1
        b.table[1, 0] = b.p.n_pages
        Q = b.random_rows(4)
        out, lse = run_attend(b, Q)
        pu.check_attend(b, Q, out, lse)


@pytest.mark.parametrize("impl", IMPLS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", mu.BLOCKS)
@pytest.mark.parametrize("d,pairs", [(64, [(1, 70), (6, 50), (40, 170), (3, 1)]), (128, [(1, 70), (6, 50), (40, 170), (3, 1)]), (128, [(150, 700), (129, 140)]),
                                     (128, [(8, 100), (1, 33)]), (128, [(30, 333), (2, 33)]), (256, [(30, 90), (2, 33)])])
def test_attention_does_not_see_what_is_hidden(dtype, form, impl, d, pairs):
    """NaN codes in the rest of a block, NaN scales in blocks that hold nothing, both in other pages, change nothing, bit for bit; NaN at a later
    position reaches the rows from it on alone."""
    say(f"hidden places dtype={dtype} form={form} impl={impl} d={d} {pairs}")
    b = mu.Batch(pairs, H=2, G=2, d=d, ps=32, block=16, dtype=dtype, form=form, impl=impl)
    Q = b.random_rows(4)
    clean, clean_lse = run_attend(b, Q)
    pu.check_attend(b, Q, clean, clean_lse)
    used = torch.zeros(b.p.n_pages, b.ps, dtype=torch.bool)
    for s, (_, n) in enumerate(b.pairs):
        for j in range(n):
            used[b.place(s, j)] = True
    nothing = ~used.view(b.p.n_pages, 2, 16).any(-1)
    for n in "KV":
        b.pool[n].view(torch.uint8).transpose(1, 2)[~used] = 0x7f
        b.pool[n + "s"].transpose(1, 2)[nothing] = math.nan
    out, lse = run_attend(b, Q)
    assert torch.equal(out, clean) and torch.equal(lse, clean_lse)
    # scales of blocks that some rows see nothing of: no influence on those, whatever their bits
    s = len(pairs) - 2
    n, length = pairs[s]
    begin = -(-(length - n + 1) // 16) * 16       # the first block behind the first row's position
    assert begin < length
    scales = {k: b.pool[k].clone() for k in ("Ks", "Vs")}
    for value in (math.nan, math.inf):
        for j in range(begin, length, 16):
            page, at = b.place(s, j)
            b.pool["Ks"][page, :, at // 16] = value
            b.pool["Vs"][page, :, at // 16] = value
        out, lse = run_attend(b, Q)
        for r, owner, pos in b.each_row():
            if owner != s or pos < begin:
                assert torch.equal(out[r], clean[r]) and torch.equal(lse[r], clean_lse[r]), (r, owner, pos, value)
            elif math.isnan(value):
                assert torch.isnan(out[r]).all(), (r, owner, pos)
    b.pool.update(scales)
    if form == gk.PAGES_INT8_BLOCKS:
        return
    late = length - n // 2
    page, at = b.place(s, late)
    b.pool["V"].view(torch.uint8)[page, :, at, 5] = 0x7f
    out, lse = run_attend(b, Q)
    assert torch.equal(lse, clean_lse)
    rest = [c for c in range(d) if c != 5]
    for r, owner, pos in b.each_row():
        if owner != s or pos < late:
            assert torch.equal(out[r], clean[r]), (r, owner, pos)
        else:
            assert torch.isnan(out[r][:, 5]).all() and (out[r][:, rest].float() - clean[r][:, rest].float()).abs().max() < 0.1


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", mu.BLOCKS)
@pytest.mark.parametrize("shape", range(len(OTHERS)))
def test_attention_does_not_depend_on_other_rows(dtype, form, shape):
    """Other queries of the later rows, and other values at positions that only they see, leave the earlier rows' bits as they are."""
    pairs, G, d = OTHERS[shape]
    say(f"other rows dtype={dtype} form={form} {pairs} G={G} d={d}")
    (n, length), = pairs
    b = mu.Batch(pairs + [(1, 32)], H=2, G=G, d=d, ps=32, block=32, dtype=dtype, form=form, seed=shape, table_pages=4096)
    b.len[1] = 4096 * 32   # (beside a long sequence a workgroup's stretch holds several tiles of the first one)
    Q = b.random_rows(2 * G)
    clean, clean_lse = run_attend(b, Q)
    late = length - n + n // 2
    other = Q.clone()
    other[n // 2:n] *= 7
    page, at = b.place(0, late)
    code = b.pool["K"].view(torch.uint8)
    for j in range(late, length):
        page, at = b.place(0, j)
        code[page, :, at, ::3] = 0x7e if form == gk.PAGES_FP8_BLOCKS else 0x7f      # the largest code
    out, lse = run_attend(b, other)
    assert torch.equal(out[:n // 2], clean[:n // 2]) and torch.equal(lse[:n // 2], clean_lse[:n // 2])
    assert not torch.equal(lse[n // 2:n], clean_lse[n // 2:n])


def dense_check(b, Q, out, lse):
    """As pu.check_attend, a sequence and head at a time."""
    out, lse = out.cpu().double(), lse.cpu().double()
    k, v, c, u = b.values("K"), b.values("V"), 1 / math.sqrt(b.d), 2.0 ** -24
    for s, (n, length) in enumerate(b.pairs):
        pages = b.table[s, :-(-length // b.ps)].long()
        r0 = int(b.start[s])
        last = torch.full((n,), length - 1) if b.cross else torch.arange(length - n, length)
        for h in range(b.H * b.G):
            kk, vv = (x[pages, h // b.G].reshape(-1, b.d)[:length] for x in (k, v))
            q = Q[r0:r0 + n, h].double()
            x = (q @ kk.T * c).masked_fill(torch.arange(length)[None] > last[:, None], -math.inf)
            w = torch.softmax(x, 1)
            want, want_lse = w @ vv, torch.logsumexp(x, 1)
            # logits, sums, weights and results, each with its rounding
            off = (b.d + 8) * u * (q.abs() @ kk.abs().T).amax(1) * c
            terms = (length + b.d + 64) * u
            weights = pu.half_step(torch.bfloat16) if b.dtype == gk.BF16 else 0.0
            bound = (w @ vv.abs()) * (weights + 4 * off + 4 * terms)[:, None] + want.abs() * pu.half_step(b.p.torch_dtype)
            assert ((out[r0:r0 + n, h] - want).abs() <= bound).all(), (s, h)
            assert ((lse[r0:r0 + n, h] - want_lse).abs() <= 2 * off + 2 * terms + want_lse.abs() * 8 * u).all(), (s, h)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", mu.BLOCKS)
@pytest.mark.parametrize("shape", range(len(LONG)))
def test_attention_over_many_parts(dtype, form, shape):
    """Long sequences of few heads, whose keys are shared out among many workgroups and joined from as many parts."""
    pairs, H, G, d = LONG[shape]
    say(f"many parts dtype={dtype} form={form} {LONG[shape]}")
    b = mu.Batch(pairs, H=H, G=G, d=d, ps=64, block=(16, 32, 64)[shape % 3], dtype=dtype, form=form, seed=shape, before=1, behind=1)
    Q = b.random_rows(H * G)
    out, lse = run_attend(b, Q)
    dense_check(b, Q, out, lse)


def test_long_offsets():
    """Places of codes beyond 2^31 bytes, and their scales."""
    say("long offsets")
    H, d, ps, block = 1, 512, 1024, 64
    p = gk.PagedParams(n_kv_heads=H, n_q_heads=H, head_dim=d, page_tokens=ps, n_pages=4200, n_seqs=1, table_pages=2, n_rows=100, max_rows=100,
                       page_format=gk.PAGES_FP8_BLOCKS, scale_tokens=block)
    pool = [torch.zeros(p.n_pages, H, ps, d, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)]
    scales = [torch.zeros(p.n_pages, H, ps // block, device="cuda") for _ in range(2)]
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    g = torch.Generator().manual_seed(1)
    batch = (i32(4199, 4198).view(1, 2), i32(1074), i32(0, 100))
    rows = [torch.randn(100, H, d, generator=g).to(torch.bfloat16) for _ in range(3)]
    gk.graphkv_cache_write(p, rows[0].cuda(), rows[1].cuda(), *pool, *batch, *scales)
    K, V = gk.graphkv_cache_read(p, *pool, *batch, *scales)
    # an e4m3 code is off by at most 2^-4 of its value or half of its least step, 2^-10 of the scale, which is at most 2 max / 448
    for got, x in ((K, rows[0]), (V, rows[1])):
        x = x.double()
        allow = x.abs() * 2.0 ** -4 + 2.0 ** -10 * 2 * x.abs().max() / 448
        assert ((got.cpu().double() - x).abs() <= allow * (1 + 2.0 ** -7)).all()
    assert pool[0].view(torch.uint8)[:4198].max() == 0
    p.impl = gk.IMPL_GENERIC
    gk.graphkv_attend(p, rows[2].cuda(), *pool, *batch, *scales)
    p.impl = gk.IMPL_AUTO
    torch.cuda.synchronize()


def test_strides_and_padding():
    say("strides and padding")
    b = mu.Batch([(3, 40), (50, 90)], form=gk.PAGES_INT8_BLOCKS, H=2, G=2, d=64, ps=16, before=3, behind=4)
    Q, args = on_gpu(b.random_rows(4)), b.device()
    want = gk.graphkv_attend(b.p, Q, *args)
    wide = torch.full((b.rows, 6, 96), -7.0, dtype=torch.bfloat16, device="cuda")
    gk.graphkv_attend(b.p, Q, *args, out=wide[:, 1:5, 16:80])
    assert torch.equal(wide[3:-4, 1:5, 16:80], want[3:-4])
    wide[3:-4, 1:5, 16:80] = -7
    assert (wide == -7).all()
