"""Attention of rows over all that another sequence holds, against its definition in 64 bits (GPU)."""
import math

import pytest
import torch

from paper_2509_00388_amd import binding as gk
from tests import more_util as mu
from tests import paged_util as pu
from tests.test_gpu_blocks import dense_check
from tests.test_gpu_paged import bits, on_gpu, say

pytestmark = pytest.mark.gpu

TYPES = [gk.BF16, gk.FP32]
FORMS = [gk.PAGES_PLAIN, gk.PAGES_FP8, gk.PAGES_INT8] + mu.BLOCKS
IMPLS = [gk.IMPL_AUTO, gk.IMPL_GENERIC]


def run_cross(b, Q, **kw):
    args = b.device()
    out = torch.full((b.rows, b.H * b.G, b.d), -7.0, dtype=b.p.torch_dtype, device="cuda")
    lse = torch.full((b.rows, b.H * b.G), -7.0, device="cuda")
    ws = torch.randint(0, 256, (gk.graphkv_attend_workspace_bytes(b.p),), dtype=torch.uint8, device="cuda")
    gk.graphkv_cross_attend(b.p, on_gpu(Q), *args, out=out, lse=lse, ws=ws, **kw)
    outside = torch.ones(b.rows, dtype=torch.bool)
    for r, _, _ in b.each_row():
        outside[r] = False
    assert (out.cpu()[outside] == -7).all() and (lse.cpu()[outside] == -7).all()
    return out, lse


SHAPES = [
    # single tokens over states of every length, none and one among them
    dict(pairs=[(1, 1)], H=1, G=1, d=128), dict(pairs=[(1, 129), (1, 0), (1, 1), (1, 512)], H=2, G=4, d=128, ps=64),
    dict(pairs=[(1, 700), (1, 64)], H=3, G=7, d=64, ps=32), dict(pairs=[(1, 300)] * 5, H=2, G=32, d=80, ps=16),
    # more rows than states
    dict(pairs=[(8, 3), (30, 1), (1, 250), (4, 0)], H=2, G=4, d=128, ps=64), dict(pairs=[(100, 7), (70, 64), (90, 65)], H=2, G=2, d=64),
    dict(pairs=[(300, 129), (129, 0), (1, 64), (260, 1)], H=1, G=2, d=128, ps=32),
    # prompts
    dict(pairs=[(100, 300)], H=2, G=4, d=128), dict(pairs=[(33, 33)], H=3, G=1, d=64, ps=32),
    dict(pairs=[(1, 150), (70, 200), (8, 90), (129, 130)], H=2, G=2, d=128, ps=32), dict(pairs=[(150, 700), (260, 333)], H=1, G=2, d=96, ps=64),
    dict(pairs=[(1, 150), (70, 200), (8, 90), (129, 130), (1, 1), (1, 33), (2, 64), (0, 9), (1, 400)], H=2, G=2, d=128, ps=32),
    # other head dimensions, groups and pages
    dict(pairs=[(1, 200), (40, 140)], H=2, G=2, d=256), dict(pairs=[(3, 120)], H=2, G=2, d=160, ps=64),
    dict(pairs=[(2, 90), (20, 60)], H=1, G=2, d=512), dict(pairs=[(1, 100), (45, 45)], H=2, G=1, d=16), dict(pairs=[(1, 140)], H=1, G=48, d=64),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_cross_attention(dtype, form, shape):
    say(f"cross attention dtype={dtype} form={form} {SHAPES[shape]}")
    b = mu.Batch(cross=True, dtype=dtype, form=form, before=1, behind=2, seed=shape, **SHAPES[shape])
    Q = b.random_rows(b.H * b.G, fused=2 * b.H)
    out, lse = run_cross(b, Q)
    pu.check_attend(b, Q, out, lse)


@pytest.mark.parametrize("form,ps", [(gk.PAGES_PLAIN, 1), (gk.PAGES_PLAIN, 2), (gk.PAGES_FP8, 4), (gk.PAGES_INT8, 8)])
def test_small_pages(form, ps):
    say(f"cross attention form={form} ps={ps}")
    for pairs in ([(1, 60), (2, 33)], [(40, 90)], [(160, 90)]):
        b = mu.Batch(pairs, cross=True, form=form, H=2, G=1, d=64, ps=ps, before=1, behind=1)
        Q = b.random_rows(2)
        out, lse = run_cross(b, Q)
        pu.check_attend(b, Q, out, lse)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", FORMS)
def test_scalar_kernel(dtype, form):
    say(f"cross attention, scalar kernel dtype={dtype} form={form}")
    b = mu.Batch([(1, 400), (30, 300), (4, 2), (3, 0)], cross=True, H=2, G=2, d=80, ps=32, block=32, dtype=dtype, form=form, impl=gk.IMPL_GENERIC,
                 before=1, behind=1)
    Q = b.random_rows(4)
    out, lse = run_cross(b, Q)
    pu.check_attend(b, Q, out, lse)


@pytest.mark.parametrize("impl", IMPLS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", FORMS)
def test_hidden_places(dtype, form, impl):
    """Infinities and NaN in the rest of a page and in other pages change nothing; pages that are none hold nothing."""
    say(f"cross attention, hidden places dtype={dtype} form={form} impl={impl}")
    for d, pairs in ((64, [(1, 70), (6, 50), (40, 170), (3, 1)]), (128, [(150, 700), (129, 40)]), (128, [(1, 70), (8, 50)])):
        b = mu.Batch(pairs, cross=True, H=2, G=2, d=d, ps=32, dtype=dtype, form=form, impl=impl)
        b.table[0, 1] = -1
        b.table[1, 0] = b.p.n_pages
        Q = b.random_rows(4)
        clean, clean_lse = run_cross(b, Q)
        pu.check_attend(b, Q, clean, clean_lse)
        used = torch.zeros(b.p.n_pages, b.ps, dtype=torch.bool)
        for s, (_, n) in enumerate(b.pairs):
            for j in range(n):
                if b.place(s, j):
                    used[b.place(s, j)] = True
        nothing = ~used.view(b.p.n_pages, -1, 16).any(-1)
        for n in "KV":
            if form == gk.PAGES_PLAIN:
                b.pool[n].transpose(1, 2)[~used] = math.nan
                b.pool[n].transpose(1, 2)[tuple((~used).nonzero()[::3].T)] = math.inf
            else:
                b.pool[n].view(torch.uint8).transpose(1, 2)[~used] = 0x7f
                b.pool[n + "s"].transpose(1, 2)[nothing if form in mu.BLOCKS else ~used] = math.nan
        out, lse = run_cross(b, Q)
        assert torch.equal(out, clean) and torch.equal(lse, clean_lse)


@pytest.mark.parametrize("impl", IMPLS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pairs,G,d", [([(1, 1)], 4, 64), ([(1, 300), (8, 90)], 4, 128), ([(1, 40), (2, 30)], 2, 256), ([(12, 300), (3, 40)], 4, 128),
                                       ([(30, 200)], 4, 64), ([(90, 400), (30, 60)], 4, 128)])
def test_infinite_values_and_logits(dtype, impl, pairs, G, d):
    """Infinite values are infinities of their sign in all rows, in their column alone; keys with logits of -infinity weigh nothing."""
    say(f"cross attention, infinite values dtype={dtype} impl={impl} {pairs} G={G} d={d}")
    b = mu.Batch(pairs, cross=True, H=2, G=G, d=d, ps=16, dtype=dtype, impl=impl, before=1, behind=1)
    Q = b.random_rows(2 * G)
    finite = b.pool["V"].clone()
    odd = {}
    for s, (n, length) in enumerate(pairs):
        for j, column, sign in ((0, 3, 1), (length // 3, 20, -1), (length - 1, 40, 1)):
            page, at = b.place(s, j)
            b.pool["V"][page, :, at, column] = sign * math.inf
            finite[page, :, at, column] = 0
            odd[s, column] = sign
    out, lse = run_cross(b, Q)
    b.pool["V"] = finite
    want, want_lse, bound, lse_bound = b.attend(Q)
    out, lse = out.cpu().double(), lse.cpu().double()
    for r, s, _ in b.each_row():
        rest = torch.ones(d, dtype=torch.bool)
        for (owner, column), sign in odd.items():
            if owner == s:
                assert (out[r, :, column] == sign * math.inf).all(), (r, s)
                rest[column] = False
        assert ((out[r] - want[r]).abs() <= bound[r] + 2.0 ** -100)[:, rest].all(), (r, s)
        assert ((lse[r] - want_lse[r]).abs() <= lse_bound[r]).all(), (r, s)
    Q[:, :, 7] = 1.5
    hidden = pairs[0][1] // 2
    for j in range(hidden):
        page, at = b.place(0, j)
        b.pool["K"][page, :, at, 7] = -math.inf
    out, lse = run_cross(b, Q)
    cell = b.place
    b.place = lambda s, pos: None if s == 0 and pos < hidden else cell(s, pos)
    b.pool["K"] = b.pool["K"].clone()
    pu.check_attend(b, Q, out, lse)


LONG = [([(1, 20000), (1, 30)], 1, 4, 128), ([(1, 70000)], 2, 1, 64), ([(12, 9000)], 1, 4, 128), ([(60, 12000), (5, 3000)], 1, 4, 128),
        ([(300, 4100)], 2, 1, 64), ([(700, 2500)], 1, 1, 128), ([(40, 5000)], 1, 4, 256), ([(1, 4000)] * 8 + [(200, 7000)], 1, 2, 128)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("shape", range(len(LONG)))
def test_many_parts(dtype, form, shape):
    pairs, H, G, d = LONG[shape]
    say(f"cross attention, many parts dtype={dtype} form={form} {LONG[shape]}")
    b = mu.Batch(pairs, cross=True, H=H, G=G, d=d, ps=64, block=(16, 64, 32)[shape % 3], dtype=dtype, form=form, seed=shape, before=1, behind=1)
    Q = b.random_rows(H * G)
    out, lse = run_cross(b, Q)
    dense_check(b, Q, out, lse)


@pytest.mark.parametrize("dtype", TYPES)
def test_many_sequences(dtype):
    say(f"cross attention, many sequences dtype={dtype}")
    g = torch.Generator().manual_seed(11)
    pairs = [(int(torch.randint(0, 3, (1,), generator=g)), int(torch.randint(0, 40, (1,), generator=g))) for _ in range(300)]
    pairs[290] = (40, 60)
    b = mu.Batch(pairs, cross=True, H=1, G=2, d=64, ps=8, dtype=dtype, before=1, behind=1)
    Q = b.random_rows(2)
    out, lse = run_cross(b, Q)
    pu.check_attend(b, Q, out, lse)


@pytest.mark.parametrize("impl", IMPLS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", FORMS)
def test_a_row_over_its_own_tokens(dtype, form, impl):
    """A sequence's last row sees the same positions as in causal attention: the same bits where each sequence has one row."""
    say(f"cross and causal dtype={dtype} form={form}")
    b = mu.Batch([(1, 300), (1, 1), (1, 64), (1, 1000)], H=2, G=4, d=128, ps=64, dtype=dtype, form=form, impl=impl)
    Q, args = on_gpu(b.random_rows(8)), b.device()
    lse = [torch.empty(4, 8, device="cuda") for _ in range(2)]
    want = gk.graphkv_attend(b.p, Q, *args, lse=lse[0])
    got = gk.graphkv_cross_attend(b.p, Q, *args, lse=lse[1])
    assert torch.equal(got, want) and torch.equal(lse[0], lse[1])


def test_strides_scale_and_padding():
    say("cross attention, strides")
    b = mu.Batch([(3, 40), (50, 20)], cross=True, H=2, G=2, d=64, ps=16, before=2, behind=3)
    b.p.softmax_scale = 0.3
    Q = b.random_rows(4, by_head=True)
    out, lse = run_cross(b, Q)
    want, want_lse, bound, _ = b.attend(Q, 0.3)
    mine = ~want.isnan()
    assert ((out.cpu().double() - want).abs() <= bound + 2.0 ** -100)[mine].all()
    wide = torch.full((b.rows, 6, 96), -7.0, dtype=torch.bfloat16, device="cuda")
    gk.graphkv_cross_attend(b.p, on_gpu(Q), *b.dev, out=wide[:, 1:5, 16:80])
    assert torch.equal(wide[2:-3, 1:5, 16:80], out[2:-3])
    wide[2:-3, 1:5, 16:80] = -7
    assert (wide == -7).all()


@pytest.mark.parametrize("pairs,form", [([(1, 60)] * 3 + [(1, 900)], gk.PAGES_PLAIN), ([(8, 200), (1, 40), (100, 150)], gk.PAGES_FP8_BLOCKS),
                                        ([(40, 90), (300, 70)], gk.PAGES_INT8)])
def test_captured(pairs, form):
    """A captured call, replayed with other lengths, pages and rows, with eager work between: the eager calls' bits."""
    say(f"cross attention captured {pairs} form={form}")
    b = mu.Batch(pairs, cross=True, H=2, G=2, d=128, ps=16, form=form, behind=3, table_pages=80, spare=80 * len(pairs))
    args, Q = b.device(), on_gpu(b.random_rows(4))
    ws, other = gk.alloc_attend_workspace(b.p), gk.alloc_attend_workspace(b.p)
    out = torch.zeros_like(Q)
    gk.graphkv_cross_attend(b.p, Q, *args, out=out, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gk.graphkv_cross_attend(b.p, Q, *args, out=out, ws=ws)
    g = torch.Generator().manual_seed(1)
    for n in range(5):
        args[3].copy_(torch.randint(0, 1200, args[3].shape, generator=g))
        args[2].copy_(torch.randint(0, b.p.n_pages, args[2].shape, generator=g))
        Q.copy_(torch.randn(Q.shape, generator=g))
        out.fill_(-7)
        graph.replay()
        got = out.clone()
        want = torch.full_like(out, -7)
        gk.graphkv_cross_attend(b.p, Q, *args, out=want, ws=other)
        assert torch.equal(bits(got), bits(want)), n
        torch.cuda.synchronize()


def test_two_streams():
    say("cross attention, two streams")
    sets = []
    for seed, pairs in ((1, [(1, 3000)]), (2, [(60, 500), (300, 700)])):
        b = mu.Batch(pairs, cross=True, H=2, G=4, d=128, ps=16, seed=seed)
        Q, args = on_gpu(b.random_rows(8)), b.device()
        sets.append((b, Q, args, gk.alloc_attend_workspace(b.p), gk.graphkv_cross_attend(b.p, Q, *args), torch.cuda.Stream()))
    torch.cuda.synchronize()
    outs = []
    for _ in range(5):
        for b, Q, args, ws, want, stream in sets:
            with torch.cuda.stream(stream):
                outs.append((gk.graphkv_cross_attend(b.p, Q, *args, ws=ws), want))
    torch.cuda.synchronize()
    for got, want in outs:
        assert torch.equal(got, want)
