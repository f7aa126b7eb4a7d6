"""CPU-only checks of pages in blocks, of attention over another sequence's states and of pages dealt on the device: what the
calls refuse before anything touches a GPU, and the definitions that the GPU tests compare with."""
import ctypes
import math
import os

import pytest
import torch

from paper_2509_00388_amd import binding as gk
from tests import more_util as mu
from tests import paged_util as pu
from tests.test_paged_cpu import BAD, FAKE, ODD, good

BLOCK = dict(page_format=gk.PAGES_FP8_BLOCKS, scale_tokens=32)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(gk.LIB_PATH):
        from paper_2509_00388_amd import build
        build.build()
    return gk.load_library()


def calls(lib, cp, ptr=FAKE, ws=1 << 40, scales=FAKE):
    c = ctypes.byref(cp)
    return {"write": lib.graphkv_cache_write(c, ptr, ptr, ptr, ptr, scales, scales, ptr, ptr, ptr, None),
            "read": lib.graphkv_cache_read(c, ptr, ptr, scales, scales, ptr, ptr, ptr, ptr, ptr, None),
            "attend": lib.graphkv_attend(c, ptr, ptr, ptr, scales, scales, ptr, ptr, ptr, ptr, None, ptr, ws, None),
            "cross": lib.graphkv_cross_attend(c, ptr, ptr, ptr, scales, scales, ptr, ptr, ptr, ptr, None, ptr, ws, None)}


def assign(lib, cp, at=None, ptr=FAKE, rest=FAKE, ws=FAKE, size=1 << 40):
    """graphkv_cache_assign with one of its twelve arrays `ptr` and the rest `rest`."""
    arrays = [ptr if i == at else rest for i in range(11)]
    return lib.graphkv_cache_assign(ctypes.byref(cp) if cp is not None else None, *arrays, ws, size, None)


@pytest.mark.parametrize("kw", [b for b in BAD if "page_format" not in b] + [dict(page_format=4), dict(page_format=7), dict(page_format=13)])
def test_invalid_params_are_refused(lib, kw):
    p = good(**{**BLOCK, **kw})
    assert set(calls(lib, p.c()).values()) == {-1}, kw
    assert assign(lib, p.c()) == -1
    assert gk.graphkv_attend_workspace_bytes(p) == 0 and gk.graphkv_assign_workspace_bytes(p) == 0


@pytest.mark.parametrize("kw", [dict(scale_tokens=8), dict(scale_tokens=24), dict(scale_tokens=128), dict(scale_tokens=-32), dict(page_tokens=8),
                                dict(scale_tokens=1 << 30), dict(head_dim=72)])
@pytest.mark.parametrize("form", mu.BLOCKS)
def test_blocks_of_other_sizes_are_refused(lib, form, kw):
    p = good(**{**BLOCK, "page_format": form, **kw})
    assert set(calls(lib, p.c()).values()) == {-1} and assign(lib, p.c()) == -1
    assert gk.graphkv_attend_workspace_bytes(p) == 0


def test_a_scales_tokens_are_read_with_blocks_alone(lib):
    p = good()
    cp = p.c()
    cp.scale_tokens = 7
    assert lib.graphkv_attend_workspace_bytes(ctypes.byref(cp)) == gk.graphkv_attend_workspace_bytes(p) > 0
    assert good(**{**BLOCK, "scale_tokens": 0}).c().scale_tokens == 32
    assert good(**{**BLOCK, "scale_tokens": 0, "page_tokens": 16}).c().scale_tokens == 16


def test_pages_without_tokens_are_refused_as_other_params(lib):
    """The binding counts the scales of a pool before the library sees the params."""
    for kw in (dict(page_tokens=0), dict(page_tokens=0, scale_tokens=0), dict(page_tokens=-16, scale_tokens=0)):
        p = good(**{**BLOCK, **kw})
        assert p.tokens_a_scale > 0
        assert set(calls(lib, p.c()).values()) == {-1}


def test_pointers_and_workspace_are_checked(lib):
    for p in (good(), good(**BLOCK)):
        need = gk.graphkv_attend_workspace_bytes(p)
        assert need > 0
        for bad in (None, ODD):
            assert set(calls(lib, p.c(), ptr=bad).values()) == {-1}
        assert calls(lib, p.c(), ws=need - 1)["cross"] == -2 and calls(lib, p.c(), ws=need - 1)["attend"] == -2
    assert set(calls(lib, good(**BLOCK).c(), scales=None).values()) == {-1}
    for strides in ((1, 0), (1020, 128), (64, 128), (-1024, 128)):
        assert calls(lib, good().c(strides))["cross"] == -1 and calls(lib, good().c((0, 0), strides))["cross"] == -1
    for kw in (dict(n_q_heads=12), dict(softmax_scale=-1.0), dict(softmax_scale=float("nan"))):
        assert calls(lib, good(**kw).c())["cross"] == -1
    assert lib.graphkv_cross_attend(None, *[FAKE] * 11, 1 << 40, None) == -1


def test_assign_checks_its_arrays(lib):
    p = good()
    assert assign(lib, None) == -1
    odd = ctypes.c_void_p(0x10002)
    for at in range(11):
        assert assign(lib, p.c(), at, odd) == -1, at
        if at not in (0, 9, 10):       # keep, positions and slots are optional
            assert assign(lib, p.c(), at, None) == -1, at
    many = good(n_seqs=1025)
    need = gk.graphkv_assign_workspace_bytes(many)
    assert need > 0 and gk.graphkv_assign_workspace_bytes(good(n_seqs=1024)) == 0
    assert assign(lib, many.c(), size=need - 1) == -2 and assign(lib, many.c(), ws=None) == -2
    assert assign(lib, many.c(), ws=ctypes.c_void_p(0x10040)) == -2
    assert gk.graphkv_assign_workspace_bytes(good(n_seqs=1 << 20)) < 1 << 16


def test_nothing_to_do_is_no_error(lib):
    for kw in (dict(n_rows=0, max_rows=0), dict(n_seqs=0)):
        p = good(**{**BLOCK, **kw})
        assert set(calls(lib, p.c(), ptr=None, ws=0, scales=None).values()) == {0}


def test_binding_refuses_host_tensors():
    b = mu.Batch([(3, 20)], form=gk.PAGES_INT8_BLOCKS, H=2, G=2, d=32)
    x = b.random_rows(2)
    args = [b.pool["K"], b.pool["V"], b.table, b.len, b.start, b.pool["Ks"], b.pool["Vs"]]
    i32 = torch.zeros(8, dtype=torch.int32)
    for call in (lambda: gk.graphkv_cache_write(b.p, x, x, *args), lambda: gk.graphkv_cache_read(b.p, *args),
                 lambda: gk.graphkv_attend(b.p, x, *args), lambda: gk.graphkv_cross_attend(b.p, x, *args),
                 lambda: gk.graphkv_cache_assign(b.p, i32, i32, b.table, i32, i32)):
        with pytest.raises(gk.GraphKVError, match="device tensor"):
            call()


def test_definition_of_blocks():
    """Hand-worked blocks: a scale over several rows, rows added behind others, a scale that grows, one that stays."""
    b = mu.Batch([(2, 3)], form=gk.PAGES_FP8_BLOCKS, H=1, G=1, d=16, ps=16, dtype=gk.FP32, spare=0)
    b.pool["K"] = torch.zeros(1, 1, 16, 16).to(torch.float8_e4m3fn)
    b.pool["K"][0, 0, 0, :3] = torch.tensor([448.0, 17.0, 0.0625]).to(torch.float8_e4m3fn)     # (17 is stored as 16)
    b.pool["Ks"] = torch.tensor([[[1.0]]])
    b.pool["V"], b.pool["Vs"] = b.pool["K"].clone(), b.pool["Ks"].clone()
    K = torch.zeros(2, 1, 16)
    V = torch.zeros(2, 1, 16)
    K[0, 0, :2] = torch.tensor([900.0, 4.0])       # needs a scale of 4
    K[1, 0, 0] = -1800.0                           # of 8
    V[1, 0, :2] = torch.tensor([-100.0, 1.0])      # of 1/4: the scale stays 1
    got = mu.written(b, K, V)
    assert got["Ks"].tolist() == [[[8.0]]] and got["Vs"].tolist() == [[[1.0]]]
    k = got["K"].float()[0, 0]
    assert k[0, :3].tolist() == [56.0, 2.0, 2.0 ** -7]
    assert k[1, :2].tolist() == [112.0, 0.5] and k[2, 0].item() == -224.0      # (112.5 and 225 lie next to 112 and 224)
    assert got["V"].float()[0, 0, 2, :2].tolist() == [-96.0, 1.0]              # (100 lies in the middle of 96 and 104: the even code)
    # a block that begins with a new row forgets the scale that it had
    b = mu.Batch([(3, 3)], form=gk.PAGES_INT8_BLOCKS, H=1, G=1, d=16, ps=16, dtype=gk.FP32, spare=0)
    b.pool["Ks"][:] = 100.0
    K = torch.zeros(3, 1, 16)
    K[1, 0, 0], K[2, 0, 5] = 254.0, 3.0
    got = mu.written(b, K, K)
    assert got["Ks"].item() == 2.0 and got["K"][0, 0, :3].double().sum().item() == 127 + 2      # (1.5: the even code)
    # codes in blocks of one row's tokens are those of rows with a scale each
    x = torch.randn(4, 2, 1, 16, generator=torch.Generator().manual_seed(1)).double()
    for form in mu.BLOCKS:
        code, scale = pu.encode(x, mu.ROW_FORM[form])
        assert torch.equal(mu.codes(x, scale[..., None], form), code) and torch.equal(mu.scale_of(x, form), scale)


def test_definition_of_attention_over_other_states():
    b = mu.Batch([(3, 9), (2, 1), (1, 0)], cross=True, H=2, G=2, d=16, ps=4, dtype=gk.FP32, before=1, behind=1)
    Q = b.random_rows(4)
    out, lse, bound, _ = b.attend(Q)
    assert out[0].isnan().all() and out[-1].isnan().all()
    for s, (n, length) in enumerate(b.pairs):
        rows = slice(int(b.start[s]), int(b.start[s + 1]))
        if length == 0:
            assert (out[rows] == 0).all() and (lse[rows] == -math.inf).all()
            continue
        pages = b.table[s, :-(-length // 4)].long()
        for h in range(4):
            k, v = (b.values(x)[pages][:, h // 2].reshape(-1, 16)[:length] for x in "KV")
            x = Q[rows, h].double() @ k.T / 4
            assert torch.allclose(out[rows, h], torch.softmax(x, 1) @ v, rtol=1e-12, atol=1e-12)
            assert torch.allclose(lse[rows, h], torch.logsumexp(x, 1), rtol=1e-12, atol=1e-12)
    assert float(bound[1:-1].max()) < 1e-3


def test_definition_of_dealt_pages():
    """A hand-worked turn, pages of 4: one sequence grows within its page, one ends, one takes pages that came back, one is refused."""
    table = torch.tensor([[7, 0, 0], [5, 6, 9], [8, 0, 0], [4, 0, 0], [3, 0, 0]], dtype=torch.int32)
    stack = torch.tensor([1, 2, 0, 0, 0, 0, 0, 0, 0, 0], dtype=torch.int32)
    got = mu.assigned([2, 0, 4, 4, 1], [2, 0, 5, 8, 1], [2, 10, 4, 4, 4], table, stack, 2, 4, 20, 0)
    length, new_table, new_stack, n_free, start, pos, slot = got
    # 1, 2, then 9, 6, 5 (the ended sequence's, so that 5 lies on top): 5 and 6 for the third sequence, and 9 and 2 for the fourth
    assert new_stack[:5].tolist() == [1, 2, 9, 6, 5] and n_free.tolist() == [1]
    assert length.tolist() == [4, 0, 9, 12, 2] and start.tolist() == [0, 2, 2, 7, 15, 16]
    assert new_table[2].tolist() == [8, 5, 6] and new_table[3].tolist() == [4, 9, 2] and new_table[1].tolist() == [5, 6, 9]
    assert pos[:7].tolist() == [2, 3, 4, 5, 6, 7, 8] and slot[:3].tolist() == [30, 31, 20] and pos[15:].tolist() == [1, -1, -1, -1, -1]
    # with one page less the fourth is refused, and the last, which needs none, is not
    length, _, _, n_free, start, _, _ = mu.assigned([2, 0, 4, 4, 1], [2, 0, 5, 8, 1], [2, 10, 4, 4, 4], table, stack, 0, 4, 20, 0)
    assert length.tolist() == [4, 0, 9, 4, 2] and start.tolist() == [0, 2, 2, 7, 7, 8] and n_free.tolist() == [1]
    # too few rows: the third is refused, so is the fourth; the last still counts them
    length, _, _, _, start, _, _ = mu.assigned([2, 0, 4, 4, 1], [2, 0, 5, 8, 0], [2, 10, 4, 4, 4], table, stack, 2, 4, 6, 0)
    assert length.tolist() == [4, 0, 4, 4, 1] and start.tolist() == [0, 2, 2, 2, 2, 2]
