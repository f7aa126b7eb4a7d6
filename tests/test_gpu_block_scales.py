"""Attention over pages of 8-bit codes with a scale a block: scales of every size, few blocks of rows over many keys, large pools, against the
definition in 64 bits (GPU)."""
import math

import pytest
import torch

from paper_2509_00388_amd import binding as gk
from tests import more_util as mu
from tests import paged_util as pu
from tests.test_gpu_blocks import dense_check
from tests.test_gpu_cross import run_cross
from tests.test_gpu_paged import bits, run_attend, say

pytestmark = pytest.mark.gpu

TYPES = [gk.BF16, gk.FP32]
# the kernels for few rows, for blocks of 64 and of 128 of them, and for blocks of 256
PAIRS = [[(1, 300), (3, 90)], [(12, 300), (20, 90)], [(60, 300), (40, 90)], [(70, 300), (3, 90)]]


def run(b, Q):
    return (run_cross if b.cross else run_attend)(b, Q)


def check(want, out, lse):
    """What pu.check_attend checks, with a definition that is there already."""
    value, _, bound, _ = want
    mine = ~value.isnan()
    out, lse = out.double().cpu(), lse.double().cpu()
    assert torch.isfinite(out[mine]).all()
    assert ((out - value).abs() <= bound + 2.0 ** -100)[mine].all()
    check_lse(want, lse)


def check_lse(want, lse):
    _, log_sum, _, lse_bound = want
    lse = lse.double().cpu()
    none = log_sum == -math.inf
    assert (lse[none] == -math.inf).all()
    assert ((lse - log_sum).abs() <= lse_bound)[~log_sum.isnan() & ~none].all()


def some_blocks(b, share):
    """A choice among all blocks of the pool, [pages, heads, blocks of a page]."""
    return torch.rand(b.p.n_pages, b.H, b.ps // b.block, generator=b.g) < share


def sized(b, n, exponents):
    """The pool's rows with a power of two a block, of these."""
    e = torch.tensor(exponents)[torch.randint(0, len(exponents), (b.p.n_pages, b.H, b.ps // b.block), generator=b.g)].double()
    size = torch.exp2(e).repeat_interleave(b.block, 2)[..., None]
    x = b.values(n)
    b.set_pool(n, (x / x.abs().amax() * size).to(b.p.torch_dtype))


@pytest.mark.parametrize("cross", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", mu.BLOCKS)
@pytest.mark.parametrize("pairs", PAIRS)
@pytest.mark.parametrize("d", [64, 128, 256])
def test_scales_of_values_that_are_zero(cross, dtype, form, pairs, d):
    """A block of codes that are 0 adds nothing to the output and its weights to the sum, whatever its scale is."""
    say(f"scales of values that are zero cross={cross} dtype={dtype} form={form} {pairs} d={d}")
    b = mu.Batch(pairs, cross=cross, H=2, G=2, d=d, ps=32, block=16, dtype=dtype, form=form, before=1, behind=1, spare=3, seed=d)
    zero = some_blocks(b, 0.5)
    b.pool["V"].view(torch.uint8)[zero.repeat_interleave(b.block, 2)] = 0
    Q = b.random_rows(4)
    want = b.attend(Q)
    for scale in (0.0, 2.0 ** -149, 2.0 ** -130, 2.0 ** -126, 2.0 ** -108, 2.0 ** -60, 2.0 ** 60, 2.0 ** 100):
        b.pool["Vs"][zero] = scale
        check(want, *run(b, Q))


@pytest.mark.parametrize("cross", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", mu.BLOCKS)
@pytest.mark.parametrize("pairs", PAIRS)
@pytest.mark.parametrize("d", [64, 128])
def test_values_of_all_sizes(cross, dtype, form, pairs, d):
    """Blocks of values next to nothing and of large ones beside others; the logarithm of the sum does not depend on them."""
    say(f"values of all sizes cross={cross} dtype={dtype} form={form} {pairs} d={d}")
    for exponents in ((0, -90, -95, -99), (-90, -99), (0, 20, 33, -33, -20), (0, 60, 90, -60), (119, 0, 127)):
        b = mu.Batch(pairs, cross=cross, H=2, G=2, d=d, ps=32, block=16, dtype=dtype, form=form, before=1, behind=1, seed=d)
        sized(b, "V", exponents)
        Q = b.random_rows(4)
        want, got = b.attend(Q), run(b, Q)
        if max(exponents) > 100:      # (sums of such values may leave the range of 32 bits)
            check_lse(want, got[1])
        else:
            check(want, *got)


@pytest.mark.parametrize("cross", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", mu.BLOCKS)
@pytest.mark.parametrize("pairs", PAIRS)
@pytest.mark.parametrize("d", [64, 128])
def test_logits_next_to_nothing(cross, dtype, form, pairs, d):
    """Scales of keys whose product with the softmax scale is below every number of 32 bits: all keys that a row sees weigh the same."""
    say(f"logits next to nothing cross={cross} dtype={dtype} form={form} {pairs} d={d}")
    for exponents, scale in (((-99,), 2.0 ** -60), ((-99, 0), 2.0 ** -60), ((-90, 0), 2.0 ** -30)):
        b = mu.Batch(pairs, cross=cross, H=2, G=2, d=d, ps=32, block=16, dtype=dtype, form=form, before=1, behind=1, seed=d)
        sized(b, "K", exponents)
        b.p.softmax_scale = scale
        Q = b.random_rows(4)
        check(b.attend(Q, scale), *run(b, Q))


@pytest.mark.parametrize("cross", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pairs", PAIRS)
@pytest.mark.parametrize("d", [48, 64, 80, 96, 112, 128, 160, 192, 240])
def test_values_that_are_no_numbers_stay_in_their_column(cross, dtype, pairs, d):
    """NaN in one column of early values, which all rows see, over several tiles: NaN in that column alone, everything else as without."""
    say(f"NaN in a column cross={cross} dtype={dtype} {pairs} d={d}")
    b = mu.Batch(pairs, cross=cross, H=2, G=2, d=d, ps=32, block=16, dtype=dtype, form=gk.PAGES_FP8_BLOCKS, before=1, behind=1, seed=d)
    Q = b.random_rows(4)
    clean, clean_lse = run(b, Q)
    pu.check_attend(b, Q, clean, clean_lse)
    code = b.pool["V"].view(torch.uint8).clone()
    # (a tile of keys that some rows do not see all of takes such values apart from the product, with weights of 32 bits)
    tile = 256 if d <= 64 else 128
    early = [n if cross else (n - new + 1) // tile * tile for new, n in pairs]
    assert early[0] >= 128 or max(n for n, _ in pairs) > 1
    owner = torch.full((b.rows,), -1)
    for r, s, _ in b.each_row():
        owner[r] = s
    for column in sorted({0, 5, 20, d // 2, d - 9, d - 1}):
        b.pool["V"].view(torch.uint8).copy_(code)
        for s, n in enumerate(early):
            for j in range(min(n, 140)):
                page, at = b.place(s, j)
                b.pool["V"].view(torch.uint8)[page, :, at, column] = 0x7f
        out, lse = run(b, Q)
        assert torch.equal(bits(lse), bits(clean_lse)), column
        rest = [c for c in range(d) if c != column]
        assert torch.equal(out[:, :, rest], clean[:, :, rest]), column
        for s, n in enumerate(early):
            assert out[(owner == s).cuda()][:, :, column].isnan().all() == (n > 0), (column, s)


# 257 to 640 units of 256 keys of a single block of up to 64 rows a head: half of the workgroups share them
FEW_BLOCKS = [([(16, 20000)], 8, 4, 64), ([(30, 10000)], 8, 2, 128), ([(12, 8000), (12, 9000)], 8, 4, 64), ([(16, 39000)], 4, 4, 128)]


@pytest.mark.parametrize("cross,form", [(False, gk.PAGES_FP8_BLOCKS), (True, gk.PAGES_INT8_BLOCKS), (True, gk.PAGES_PLAIN), (True, gk.PAGES_FP8)])
@pytest.mark.parametrize("shape", range(len(FEW_BLOCKS)))
def test_few_blocks_over_many_keys(cross, form, shape):
    pairs, H, G, d = FEW_BLOCKS[shape]
    say(f"few blocks over many keys cross={cross} form={form} {FEW_BLOCKS[shape]}")
    b = mu.Batch(pairs, cross=cross, H=H, G=G, d=d, ps=64, block=32, form=form, seed=shape, before=1, behind=1)
    units = sum(-(-n // 256) for _, n in pairs) * H
    assert 256 < units <= 640
    Q = b.random_rows(H * G)
    out, lse = run(b, Q)
    dense_check(b, Q, out, lse)


@pytest.mark.parametrize("form", mu.BLOCKS)
@pytest.mark.parametrize("dtype,d", [(gk.BF16, 256), (gk.BF16, 128), (gk.FP32, 128)])
def test_places_beyond_two_gigabytes(form, dtype, d):
    """Codes of the pool's last pages, more than 2^31 bytes behind its begin, by every kernel, against the definition."""
    say(f"places beyond two gigabytes form={form} dtype={dtype} d={d}")
    H, ps, block = 2, 1024, 64
    pages = (1 << 31) // (H * ps * d) + 6
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    pools = [torch.zeros(pages, H, ps, d, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.zeros(pages, H, ps // block, device="cuda") for _ in range(2)]
    for cross in (False, True):
        for pairs in ([(1, 1500), (3, 700)], [(20, 1500), (12, 700)], [(150, 1300), (3, 700)]):
            b = mu.Batch(pairs, cross=cross, H=H, G=2, d=d, ps=ps, block=block, dtype=dtype, form=form, before=1, behind=1, seed=d)
            n = b.p.n_pages
            for i, name in enumerate("KV"):      # the batch's own few pages become the last of the large pools
                pools[i][-n:] = b.pool[name].view(torch.uint8).cuda()
                scales[i][-n:] = b.pool[name + "s"].cuda()
            Q, p = b.random_rows(H * 2), b.p
            want = b.attend(Q)
            p.n_pages = pages
            start, t = pages - n, b.pool["K"].dtype
            assert start * H * ps * d >= 2 ** 31
            table = b.table.cuda() + start
            out = torch.full((b.rows, H * 2, d), -7.0, dtype=p.torch_dtype, device="cuda")
            lse = torch.full((b.rows, H * 2), -7.0, device="cuda")
            call = gk.graphkv_cross_attend if cross else gk.graphkv_attend
            call(p, Q.cuda(), pools[0].view(t), pools[1].view(t), table, i32(*b.len.tolist()), i32(*b.start.tolist()), *scales, out=out, lse=lse)
            check(want, out, lse)
