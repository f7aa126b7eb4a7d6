"""CPU-only checks of the paged-cache calls: what they refuse before anything touches a GPU, sizes, and the definitions that
the GPU tests compare with."""
import ctypes
import os
import re

import pytest
import torch

from paper_2509_00388_amd import binding as gk
from tests import paged_util as pu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = ctypes.c_void_p(0x10000)
ODD = ctypes.c_void_p(0x10004)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(gk.LIB_PATH):
        from paper_2509_00388_amd import build
        build.build()
    return gk.load_library()


def good(**kw):
    p = gk.PagedParams(n_kv_heads=8, n_q_heads=32, head_dim=128, page_tokens=64, n_pages=1000, n_seqs=4, table_pages=100,
                       n_rows=40, max_rows=10)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def calls(lib, cp, ptr=FAKE, ws=1 << 40, scales=FAKE):
    """The three calls with fake but aligned pointers: checks must fail before any of them is used."""
    c = ctypes.byref(cp)
    return {"write": lib.graphkv_cache_write(c, ptr, ptr, ptr, ptr, scales, scales, ptr, ptr, ptr, None),
            "read": lib.graphkv_cache_read(c, ptr, ptr, scales, scales, ptr, ptr, ptr, ptr, ptr, None),
            "attend": lib.graphkv_attend(c, ptr, ptr, ptr, scales, scales, ptr, ptr, ptr, ptr, None, ptr, ws, None)}


def test_params_struct_layout_matches_header():
    header = open(os.path.join(ROOT, "include", "graphkv.h")).read()
    body = header.split("typedef struct graphkv_paged_params {")[1].split("} graphkv_paged_params;")[0]
    fields = re.findall(r"(int32_t|int64_t|float)\s+([a-z_]+);", re.sub(r"/\*.*?\*/", "", body, flags=re.S))
    name = {ctypes.c_float: "float", ctypes.c_int32: "int32_t", ctypes.c_int64: "int64_t"}
    assert fields == [(name[f[1]], f[0]) for f in gk._CPagedParams._fields_]


def test_kernel_ids_match_header():
    header = open(os.path.join(ROOT, "include", "graphkv.h")).read()
    ids = re.findall(r"\b(GRAPHKV_K_[A-Z_]+)\b", header.split("GRAPHKV_K_SCORE_STATS = 0")[1].split("GRAPHKV_N_KERNELS\n};")[0])
    assert len(ids) + 1 == gk.N_KERNELS
    lib = gk.load_library()
    names = [lib.graphkv_kernel_name(i).decode() for i in range(gk.N_KERNELS)]
    assert len(set(names)) == gk.N_KERNELS and "unknown" not in names
    assert names[22] == "nbr_select_later" and names[23:] == ["cache_write", "cache_read", "attend_generic", "attend_few",
                                                               "attend_many", "attend_join"]


BAD = [dict(n_kv_heads=0), dict(n_kv_heads=65536, n_q_heads=65536), dict(head_dim=0), dict(head_dim=100), dict(head_dim=520),
       dict(dtype=2), dict(page_format=3), dict(page_format=-1), dict(page_format=gk.PAGES_FP8, head_dim=72), dict(page_tokens=0),
       dict(page_tokens=48), dict(page_tokens=1 << 17), dict(n_pages=0), dict(n_pages=1 << 22), dict(n_pages=2 ** 31 - 1, page_tokens=65536, n_kv_heads=65535),
       dict(n_seqs=-1), dict(n_seqs=(1 << 20) + 1), dict(table_pages=0), dict(table_pages=1 << 25), dict(n_rows=-1),
       dict(n_rows=(1 << 26) + 1), dict(max_rows=41), dict(max_rows=-1), dict(impl=2)]


@pytest.mark.parametrize("kw", BAD)
def test_invalid_params_are_refused(lib, kw):
    got = calls(lib, good(**kw).c())
    assert set(got.values()) == {-1}, (kw, got)
    assert gk.graphkv_attend_workspace_bytes(good(**kw)) == 0


@pytest.mark.parametrize("kw", [dict(n_q_heads=0), dict(n_q_heads=12), dict(n_q_heads=65544), dict(softmax_scale=-1.0),
                                dict(softmax_scale=float("nan")), dict(softmax_scale=float("inf")),
                                dict(n_seqs=1 << 20, table_pages=1 << 20, page_tokens=1)])
def test_invalid_attention_is_refused(lib, kw):
    assert calls(lib, good(**kw).c())["attend"] == -1


@pytest.mark.parametrize("strides", [(1, 0), (1024, 4), (1020, 128), (64, 128), (1024, -128), (-1024, 128), (1 << 45, 128)])
def test_strides_are_checked(lib, strides):
    assert set(calls(lib, good().c(strides)).values()) == {-1}
    assert calls(lib, good().c((0, 0), strides))["attend"] == -1


@pytest.mark.parametrize("kw", [dict(n_rows=1 << 24), dict(n_rows=1 << 26)])
def test_rows_beyond_a_launch_are_refused(lib, kw):
    """A launch has at most 2^32 - 1 threads a dimension."""
    assert set(calls(lib, good(**kw).c()).values()) == {-1}
    assert gk.graphkv_attend_workspace_bytes(good(**kw)) == 0
    assert gk.graphkv_attend_workspace_bytes(good(n_rows=(1 << 24) - 1)) > 0


def test_sizes_that_overflow_are_refused(lib):
    """A scale whose product with log2 e is no number of 32 bits; strides whose product with the rows is none of 64."""
    assert calls(lib, good(softmax_scale=3e38).c())["attend"] == -1
    assert gk.graphkv_attend_workspace_bytes(good(softmax_scale=2.0 ** 127)) > 0
    for strides in (((1 << 38) + 8, 128), (128, (1 << 38) + 8)):
        assert set(calls(lib, good().c(strides)).values()) == {-1}


def test_outputs_must_not_overlap(lib):
    """Rows that lie within one another's heads are an output's mistake; inputs may be read that way."""
    d = 128
    p = good(n_rows=40)
    for strides in ((d, d), (4 * d, d), (4 * d, 2 * d)):
        assert calls(lib, p.c(strides))["read"] == -1
        assert calls(lib, p.c((0, 0), strides))["attend"] == -1


def test_pointers_and_workspace_are_checked(lib):
    p = good()
    need = gk.graphkv_attend_workspace_bytes(p)
    assert need > 0
    for bad in (None, ODD):
        assert set(calls(lib, p.c(), ptr=bad).values()) == {-1}
    coded = good(page_format=gk.PAGES_INT8)
    assert set(calls(lib, coded.c(), scales=None).values()) == {-1}
    assert set(calls(lib, coded.c(), scales=ctypes.c_void_p(0x10002)).values()) == {-1}
    assert calls(lib, p.c(), ws=need - 1)["attend"] == -2
    c = ctypes.byref(p.c())
    assert lib.graphkv_attend(c, FAKE, FAKE, FAKE, None, None, FAKE, FAKE, FAKE, FAKE, None, None, need, None) == -2
    assert lib.graphkv_attend(c, FAKE, FAKE, FAKE, None, None, FAKE, FAKE, FAKE, FAKE, ctypes.c_void_p(0x10001), FAKE, need, None) == -1
    assert lib.graphkv_cache_write(None, *[FAKE] * 9, None) == -1 and lib.graphkv_attend_workspace_bytes(None) == 0


def test_nothing_to_do_is_no_error(lib):
    for kw in (dict(n_rows=0, max_rows=0), dict(n_seqs=0)):
        p = good(**kw)
        assert gk.graphkv_attend_workspace_bytes(p) == 0
        assert set(calls(lib, p.c(), ptr=None, ws=0, scales=None).values()) == {0}


def test_workspace_stays_bounded(lib):
    """Scratch memory goes with the chip, not with the cache: a long context and a large batch take no more than they need to
    share their work out."""
    for kw in (dict(), dict(table_pages=1 << 14), dict(n_seqs=1024, n_rows=1024, max_rows=1), dict(n_rows=8192, max_rows=8192),
               dict(n_rows=1 << 20, max_rows=1 << 20, n_seqs=1), dict(dtype=gk.FP32, head_dim=256)):
        assert gk.graphkv_attend_workspace_bytes(good(**kw)) < 128 << 20, kw
    assert gk.graphkv_attend_workspace_bytes(good(impl=gk.IMPL_GENERIC)) == 0


def test_binding_refuses_what_the_library_cannot_see():
    b = pu.Batch([(3, 20)], H=2, G=2, d=32)
    x = b.random_rows(2)
    args = [b.pool["K"], b.pool["V"], b.table, b.len, b.start]
    for call in (lambda: gk.graphkv_cache_write(b.p, x, x, *args), lambda: gk.graphkv_cache_read(b.p, *args),
                 lambda: gk.graphkv_attend(b.p, x, *args)):
        with pytest.raises(gk.GraphKVError, match="device tensor"):
            call()


def test_definition_of_the_codes():
    """Hand-worked rows: scales and codes of both 8-bit forms."""
    x = torch.tensor([[448.0, 1.0, -17.0, 0.0], [449.0, -224.0, 3.0, 0.5], [1.75, 0.875, -1.0, 0.001953125], [0.0, 0.0, -0.0, 0.0],
                      [1.0, 2.0 ** -12, 2.0 ** -30, -1.0]])
    code, s = pu.encode(x, gk.PAGES_FP8)
    assert s.tolist() == [1.0, 2.0, 2.0 ** -8, 0.0, 2.0 ** -8]
    assert code[0].tolist() == [448.0, 1.0, -16.0, 0.0]                   # 17 lies between 16 and 18: the even code
    assert code[1].tolist() == [224.0, -112.0, 1.5, 0.25]                 # 224.5 between 224 and 240
    assert code[2].tolist() == [448.0, 224.0, -256.0, 0.5]
    assert code[3].tolist() == [0.0] * 4
    assert code[4].tolist() == [256.0, 0.0625, 0.0, -256.0]
    code, s = pu.encode(torch.tensor([[127.0, 63.5, -0.5, 1.5], [254.0, 1.0, 3.0, -254.0], [1.0, 0.5, 0.25, 0.0]]), gk.PAGES_INT8)
    assert s[:2].tolist() == [1.0, 2.0] and code[0].tolist() == [127.0, 64.0, 0.0, 2.0]
    assert code[1].tolist() == [127.0, 0.0, 2.0, -127.0]
    third = torch.tensor(1.0).double() / 127
    assert s[2] == third.float().double() and code[2, 0] == 127 and code[2, 3] == 0


def test_definition_of_attention():
    """The 64-bit attention of the tests against a softmax over a dense cache with an explicit mask."""
    b = pu.Batch([(3, 9), (1, 4)], H=2, G=2, d=16, ps=4, dtype=gk.FP32, before=1, behind=1)
    Q = b.random_rows(4)
    out, lse, bound, _ = b.attend(Q)
    assert out[0].isnan().all() and out[-1].isnan().all()
    for s, (n, length) in enumerate(b.pairs):
        pages = b.table[s, :-(-length // 4)].long()
        for h in range(4):
            k, v = (b.values(x)[pages][:, h // 2].reshape(-1, 16)[:length] for x in "KV")
            q = Q[int(b.start[s]):int(b.start[s + 1]), h].double()
            hidden = torch.arange(length)[None] > torch.arange(length - n, length)[:, None]
            x = (q @ k.T / 4).masked_fill(hidden, -torch.inf)
            rows = slice(int(b.start[s]), int(b.start[s + 1]))
            assert torch.allclose(out[rows, h], torch.softmax(x, 1) @ v, rtol=1e-12, atol=1e-12)
            assert torch.allclose(lse[rows, h], torch.logsumexp(x, 1), rtol=1e-12, atol=1e-12)
    assert float(bound[1:-1].max()) < 1e-3


@pytest.mark.parametrize("kw", [dict(n_kv_heads=64, n_q_heads=256, n_pages=1000, page_tokens=1024, table_pages=1 << 20),
                                dict(n_kv_heads=128, n_q_heads=128, n_seqs=7, n_rows=400, max_rows=100, page_tokens=1, table_pages=1 << 30),
                                dict(n_kv_heads=1, n_q_heads=64, n_rows=1 << 24, max_rows=0, n_seqs=1),
                                dict(n_kv_heads=8, n_q_heads=8, n_rows=1 << 20, max_rows=1, n_seqs=1 << 20, table_pages=255)])
def test_sizes_up_to_the_stated_limits_are_taken(lib, kw):
    """Long tables beside rows that only the kernels for many rows take, the most stacked rows, the most sequences."""
    if kw.get("n_rows") == 1 << 24:
        kw = dict(kw, n_rows=(1 << 24) - 1)
    p = good(**kw)
    G = p.n_q_heads // p.n_kv_heads
    most = p.max_rows or p.n_rows
    assert p.n_rows * G <= 1 << 30 and p.n_rows * p.n_q_heads + 192 * p.n_seqs * p.n_kv_heads < 1 << 35
    if most * G <= 32 or p.n_seqs >= 8:
        assert p.n_seqs * p.n_kv_heads * -(-p.table_pages * p.page_tokens // 128) < 1 << 31
    need = gk.graphkv_attend_workspace_bytes(p)
    assert 0 < need < 256 << 20
    assert lib.graphkv_attend(ctypes.byref(p.c()), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, need - 1, None) == -2


@pytest.mark.parametrize("kw", [dict(n_kv_heads=1, n_q_heads=128, n_rows=(1 << 23) + 1),
                                dict(n_kv_heads=8, n_q_heads=8, n_rows=1 << 20, max_rows=1, n_seqs=1 << 20, table_pages=513, page_tokens=64)])
def test_sizes_beyond_the_stated_limits_are_refused(lib, kw):
    p = good(**kw)
    assert gk.graphkv_attend_workspace_bytes(p) == 0 and calls(lib, p.c())["attend"] == -1
