"""The paged cache's refusals, on the host before anything is launched: every call below has fake device addresses and must
come back with its error (or do nothing) without touching them."""
import ctypes

import pytest
import torch

import paper_2601_21896_b200 as pafu
from paper_2601_21896_b200 import binding as B
from paper_2601_21896_b200 import build as pbuild

FAKE = 0x7f0000000000
GB = 1 << 30
INVALID, BUDGET, SHAPE, SMALL, MISALIGNED = 1, 2, 3, 4, 5


@pytest.fixture(scope="module")
def L():
    pbuild.build_library()
    return B.lib()


def cache(**kw):
    """16 pages of 32 tokens, 8 query heads over 2 key heads of 128, bf16, stored token by token; 4 requests."""
    c = B.CPagedCache(8, 2, 128, 0, 0, 32, 8, 4, 16, 32 * 256, 256, 128, FAKE, FAKE + GB, None, None, FAKE + 2 * GB)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def test_struct_layout_matches_header():
    assert ctypes.sizeof(B.CPagedCache) == 8 * 4 + 4 * 8 + 5 * 8


BAD_CACHES = [
    (INVALID, dict(n_heads=0)), (INVALID, dict(n_kv_heads=0)), (INVALID, dict(n_heads=9)), (INVALID, dict(d_head=0)),
    (INVALID, dict(type=2, cache_type=2)), (INVALID, dict(type=0, cache_type=1)), (INVALID, dict(cache_type=3)), (INVALID, dict(type=-1)),
    (INVALID, dict(page_size=0)), (INVALID, dict(max_pages=0)), (INVALID, dict(n_requests=-1)), (INVALID, dict(n_pages=0)),
    (INVALID, dict(page_stride=-256)), (INVALID, dict(token_stride=260)), (INVALID, dict(head_stride=4)),
    (INVALID, dict(cache_type=2, head_stride=136)),            # 16 bytes are 16 elements there
    (INVALID, dict(k_scale=FAKE + 3 * GB)),                    # a scale without 8-bit pools
    (INVALID, dict(K=None)), (INVALID, dict(V=None)), (INVALID, dict(table=None)),
    (SHAPE, dict(d_head=96)), (SHAPE, dict(n_heads=65538)), (SHAPE, dict(page_size=1 << 28)), (SHAPE, dict(n_pages=1 << 27)),
    (SHAPE, dict(n_pages=1 << 32, page_size=1)), (SHAPE, dict(page_stride=1 << 62)), (SHAPE, dict(page_stride=1 << 35)),
    (MISALIGNED, dict(K=FAKE + 8)), (MISALIGNED, dict(V=FAKE + 2)), (MISALIGNED, dict(table=FAKE + 2)),
    (MISALIGNED, dict(cache_type=2, v_scale=FAKE + 1)),
]


def tables(L, c, n_slots=64, ws=FAKE + 40 * GB, nb=GB, **kw):
    a = dict(old=FAKE + 3 * GB, new=FAKE + 4 * GB, free=FAKE + 5 * GB, nf=FAKE + 6 * GB, nfo=FAKE + 6 * GB, out=FAKE + 3 * GB,
             slots=FAKE + 7 * GB, cu=FAKE + 8 * GB)
    a.update(kw)
    return L.pafu_paged_tables(None if c is None else ctypes.byref(c), a["old"], a["new"], a["free"], a["nf"], a["nfo"], a["out"],
                               a["slots"], n_slots, a["cu"], ws, nb, None)


def append(L, c, n=5, ws=FAKE + 40 * GB, nb=GB, **kw):
    a = dict(K=FAKE + 10 * GB, V=FAKE + 11 * GB, ld=256, lh=128, slots=FAKE + 7 * GB)
    a.update(kw)
    return L.pafu_paged_append(None if c is None else ctypes.byref(c), a["K"], a["V"], a["ld"], a["lh"], a["slots"], n, ws, nb, None)


def attn(L, c, ws=FAKE + 40 * GB, nb=GB, **kw):
    a = dict(Q=FAKE + 12 * GB, ld=1024, lh=128, lens=FAKE + 3 * GB, sink=0, recent=-1, scale=0.0, O=FAKE + 13 * GB, LSE=FAKE + 14 * GB)
    a.update(kw)
    return L.pafu_paged_attn(None if c is None else ctypes.byref(c), a["Q"], a["ld"], a["lh"], a["lens"], a["sink"], a["recent"],
                             a["scale"], a["O"], a["LSE"], ws, nb, None)


@pytest.mark.parametrize("status,change", BAD_CACHES)
def test_a_bad_cache_is_refused_by_every_call(L, status, change):
    c = cache(**change)
    assert L.pafu_paged_workspace_bytes(ctypes.byref(c)) == 0
    assert tables(L, c) == append(L, c) == attn(L, c) == status


def test_a_missing_cache_is_refused(L):
    assert L.pafu_paged_workspace_bytes(None) == 0
    assert tables(L, None) == append(L, None) == attn(L, None) == INVALID


def test_workspace_is_checked(L):
    c = cache()
    need = L.pafu_paged_workspace_bytes(ctypes.byref(c))
    assert need > 12800 and need % 256 == 0
    for call in (tables, append, attn):
        assert call(L, c, ws=None) == INVALID
        assert call(L, c, ws=FAKE + 40 * GB + 64) == MISALIGNED
        assert call(L, c, nb=need - 1) == SMALL


def test_tables_refuse_on_the_host(L):
    c, F = cache(), FAKE
    for name in ("old", "new", "free", "nf", "nfo", "out", "slots", "cu"):
        assert tables(L, c, **{name: None}) == INVALID, name
        assert tables(L, c, **{name: F + 30 * GB + (4 if name == "slots" else 2)}) == MISALIGNED, name
    assert tables(L, c, n_slots=-1) == INVALID
    assert tables(L, c, n_slots=1 << 31) == SHAPE
    # outputs over inputs or one another, beyond the updates in place
    assert tables(L, c, out=F + 3 * GB + 8) == INVALID
    assert tables(L, c, nfo=F + 3 * GB) == INVALID
    assert tables(L, c, cu=F + 4 * GB) == INVALID
    assert tables(L, c, slots=F + 8 * GB) == INVALID
    assert tables(L, c, free=F + 2 * GB + 4) == INVALID                     # inside the block table
    assert tables(L, c, slots=F + 2 * GB) == INVALID
    assert tables(L, c, nf=F + 5 * GB, nfo=F + 9 * GB) == INVALID           # the count inside the list


def test_append_refuses_on_the_host(L):
    c = cache()
    assert append(L, c, n=0) == 0
    assert append(L, c, n=-1) == INVALID
    assert append(L, c, n=1 << 30) == SHAPE
    for name in ("K", "V", "slots"):
        assert append(L, c, **{name: None}) == INVALID
        assert append(L, c, **{name: FAKE + 30 * GB + 4}) == MISALIGNED
    assert append(L, c, ld=-256) == INVALID and append(L, c, ld=260) == INVALID and append(L, c, lh=4) == INVALID
    assert append(L, c, ld=1 << 41) == SHAPE
    pool = 16 * 32 * 256 * 2
    assert append(L, c, K=FAKE + pool - 512) == INVALID                      # rows inside the pools
    assert append(L, c, V=FAKE + GB) == INVALID
    assert append(L, c, V=FAKE + GB - 256) == INVALID
    assert append(L, cache(V=FAKE)) == INVALID                               # one pool for keys and values


def test_attention_refuses_on_the_host(L):
    c = cache()
    assert attn(L, cache(n_requests=0, table=None)) == 0
    for name in ("Q", "lens", "O"):
        assert attn(L, c, **{name: None}) == INVALID
    for name in ("Q", "O"):
        assert attn(L, c, **{name: FAKE + 30 * GB + 8}) == MISALIGNED
    assert attn(L, c, lens=FAKE + 30 * GB + 2) == MISALIGNED and attn(L, c, LSE=FAKE + 30 * GB + 2) == MISALIGNED
    assert attn(L, c, ld=1020) == INVALID and attn(L, c, lh=-128) == INVALID
    assert attn(L, c, sink=-1) == BUDGET
    for scale in (-1.0, float("nan"), float("inf")):
        assert attn(L, c, scale=scale) == INVALID
    assert attn(L, cache(n_requests=1 << 20, n_heads=4096)) == SHAPE
    assert attn(L, c, O=FAKE + 12 * GB) == INVALID                            # over the queries
    assert attn(L, c, LSE=FAKE + 13 * GB + 64) == INVALID                     # inside the output
    assert attn(L, c, O=FAKE + 1024) == INVALID                               # inside the pools
    assert attn(L, c, O=FAKE + 2 * GB) == INVALID                             # over the block table
    assert attn(L, c, LSE=FAKE + 3 * GB + 12) == INVALID                      # over the lengths


def test_binding_refuses_tensors_of_the_wrong_kind(L):
    K = torch.zeros((3, 8, 2, 64), dtype=torch.bfloat16)
    table = torch.zeros((2, 4), dtype=torch.int32)
    ok = pafu.PagedCache(K, K.clone(), table, 4)
    assert (ok.c.n_kv_heads, ok.c.page_size, ok.c.max_pages, ok.c.n_requests, ok.c.n_pages) == (2, 8, 4, 2, 3)
    for args, kw in [((K, K[:2], table, 4), {}), ((K, K.half(), table, 4), {}), ((K.float(), K.float(), table, 4), {}), ((K[0], K[0], table, 4), {}),
                     ((K, K.clone(), table.long(), 4), {}), ((K, K.clone(), table.t(), 4), {}), ((K, K.clone(), table, 4), dict(dtype=torch.float16)),
                     ((K, K.clone().transpose(1, 2).contiguous().transpose(1, 2), table, 4), {}),      # laid out differently
                     ((K, K.clone(), table, 4), dict(k_scale=torch.ones(3))), ((K, K.clone(), table, 4), dict(v_scale=torch.ones(2).half()))]:
        with pytest.raises(pafu.PafuError) as e:
            pafu.PagedCache(*args, **kw)
        assert e.value.status == INVALID
    # tensors that do not lie on a GPU
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    with pytest.raises(pafu.PafuError):
        pafu.pafu_paged_attn(ok, q, torch.zeros(2, dtype=torch.int32), q.clone(), None, ws=torch.zeros(1 << 20, dtype=torch.uint8))
