"""CPU-side checks of the entry points over pages: every argument the header rules out is refused on the host, before any launch.
Addresses below stand for device memory that no call gets to."""
import ctypes as C
import os

import pytest

from paper_2410_13344_amd import binding as B

ARG, SHAPE, CAPACITY = -1, -2, -3
A = 4096            # a 256-byte aligned stand-in for an address


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(B.LIB_PATH):
        from paper_2410_13344_amd.build import build_library
        build_library()
    return B.lib()


def pages(**kw):
    f = dict(k=A, v=A, bounds=A, n_pages=8, page_size=16, n_kv_heads=2, head_dim=64, dtype=B.CERBERUS_BF16)
    f.update(kw)
    return B.Pages(*[f[n] for n, _ in B.Pages._fields_])


def table(**kw):
    f = dict(block_table=A, kv_len=A, free_pages=A, n_free=A, status=A, max_seqs=4, max_blocks=8, page_size=16, n_pages=8)
    f.update(kw)
    return B.PageTable(*[f[n] for n, _ in B.PageTable._fields_])


def refused(L, code, rc, word):
    assert rc == code, (rc, L.cerberus_last_error())
    assert word.encode() in L.cerberus_last_error(), L.cerberus_last_error()


BAD_PAGES = [(SHAPE, dict(page_size=8), "page_size"), (SHAPE, dict(page_size=48), "page_size"), (SHAPE, dict(page_size=512), "page_size"),
             (SHAPE, dict(head_dim=96), "head_dim"), (ARG, dict(dtype=2), "dtype"), (SHAPE, dict(n_pages=0), "n_pages"),
             (SHAPE, dict(n_pages=1 << 28), "n_pages"), (SHAPE, dict(n_kv_heads=0), "n_kv_heads"), (ARG, dict(k=None), "pool"),
             (ARG, dict(v=A + 8), "aligned"), (ARG, dict(bounds=A + 4), "aligned")]
BAD_TABLES = [(ARG, dict(block_table=None), "null"), (ARG, dict(kv_len=None), "null"), (ARG, dict(free_pages=None), "null"),
              (ARG, dict(n_free=None), "null"), (ARG, dict(status=None), "null"), (SHAPE, dict(max_seqs=0), "max_seqs"),
              (SHAPE, dict(max_seqs=1025), "max_seqs"), (SHAPE, dict(max_blocks=0), "max_blocks"), (SHAPE, dict(max_blocks=1 << 28), "max_blocks"),
              (SHAPE, dict(page_size=20), "page_size"), (SHAPE, dict(n_pages=-1), "n_pages")]


@pytest.mark.parametrize("code,kw,word", BAD_PAGES)
def test_bad_pages_are_refused(L, code, kw, word):
    pg, pt = pages(**kw), table()
    refused(L, code, L.cerberus_page_store(pg, A, 128, 64, A, 128, 64, A, 3, A, None), word)
    refused(L, code, L.cerberus_page_select(pg, pt, A, 256, 2, 4, 2, A, A, 1 << 30, None), word)
    refused(L, code, L.cerberus_paged_attention(pg, pt, A, 256, A, 256, 2, 4, 0.1, None, 0, A, 1 << 30, None), word)
    assert L.cerberus_paged_workspace_bytes(pg, pt, 2, 4, 0) == 0


@pytest.mark.parametrize("code,kw,word", BAD_TABLES)
def test_bad_tables_are_refused(L, code, kw, word):
    pg, pt = pages(), table(**kw)
    refused(L, code, L.cerberus_page_plan(pt, A, 2, 16, A, A, A, None), word)
    refused(L, code, L.cerberus_page_select(pg, pt, A, 256, 2, 4, 2, A, A, 1 << 30, None), word)
    refused(L, code, L.cerberus_paged_attention(pg, pt, A, 256, A, 256, 2, 4, 0.1, None, 0, A, 1 << 30, None), word)
    assert L.cerberus_paged_workspace_bytes(pg, pt, 2, 4, 0) == 0


def test_plan_arguments(L):
    pt = table()
    for batch in (0, -1, 5):
        refused(L, ARG, L.cerberus_page_plan(pt, A, batch, 16, A, A, A, None), "batch")
    refused(L, ARG, L.cerberus_page_plan(None, A, 1, 16, A, A, A, None), "null")
    refused(L, ARG, L.cerberus_page_plan(pt, None, 1, 16, A, A, A, None), "null")
    refused(L, ARG, L.cerberus_page_plan(pt, A, 1, 16, None, A, A, None), "null")
    refused(L, ARG, L.cerberus_page_plan(pt, A, 1, 16, A, None, A, None), "null")
    refused(L, ARG, L.cerberus_page_plan(pt, A, 1, 16, A, A, None, None), "slot")
    refused(L, ARG, L.cerberus_page_plan(pt, A, 1, -1, A, A, A, None), "max_rows")


def test_store_arguments(L):
    pg = pages()
    assert L.cerberus_page_store(pg, None, 0, 0, None, 0, 0, None, 0, None, None) == 0          # no rows: nothing to do
    refused(L, ARG, L.cerberus_page_store(None, A, 128, 64, A, 128, 64, A, 3, A, None), "null")
    refused(L, ARG, L.cerberus_page_store(pg, A, 128, 64, A, 128, 64, A, -1, A, None), "n_rows")
    refused(L, ARG, L.cerberus_page_store(pg, A, 128, 64, A, 128, 64, None, 3, A, None), "slot")
    refused(L, ARG, L.cerberus_page_store(pg, None, 128, 64, A, 128, 64, A, 3, A, None), "null k")
    refused(L, ARG, L.cerberus_page_store(pg, A, 128, 64, A + 2, 128, 64, A, 3, A, None), "v and its strides")
    refused(L, ARG, L.cerberus_page_store(pg, A, 129, 64, A, 128, 64, A, 3, A, None), "k and its strides")
    refused(L, ARG, L.cerberus_page_store(pg, A, 128, 64, A, 128, 68, A, 3, A, None), "head strides")


def test_select_and_attention_arguments(L):
    pg, pt = pages(), table()
    need = L.cerberus_paged_workspace_bytes(pg, pt, 2, 4, 2)
    assert need > 0

    def select(pg=pg, pt=pt, q=A, row=256, batch=2, heads=4, n=2, blocks=A, ws=A, nbytes=need):
        return L.cerberus_page_select(pg, pt, q, row, batch, heads, n, blocks, ws, nbytes, None)

    def attend(pg=pg, pt=pt, q=A, row=256, out=A, orow=256, batch=2, heads=4, scale=0.1, blocks=A, n=2, ws=A, nbytes=need):
        return L.cerberus_paged_attention(pg, pt, q, row, out, orow, batch, heads, scale, blocks, n, ws, nbytes, None)

    for call in (select, attend):
        refused(L, ARG, call(batch=5), "batch")
        refused(L, SHAPE, call(heads=5), "n_heads")
        refused(L, SHAPE, call(heads=0), "n_heads")
        refused(L, SHAPE, call(pt=table(n_pages=9)), "differ")
        refused(L, SHAPE, call(pt=table(page_size=32)), "differ")
        refused(L, ARG, call(q=None), "null q")
        refused(L, ARG, call(q=A + 8), "16 bytes")
        refused(L, ARG, call(row=260), "16 bytes")
        refused(L, ARG, call(n=9), "n_select")
        refused(L, ARG, call(ws=None), "workspace")
        refused(L, ARG, call(ws=A + 16), "workspace")
        refused(L, CAPACITY, call(nbytes=need - 1), "workspace")
    refused(L, ARG, select(pg=pages(bounds=None)), "bounds")
    refused(L, ARG, select(n=0), "n_select")
    refused(L, ARG, select(blocks=None), "blocks")
    refused(L, ARG, attend(out=None), "null out")
    refused(L, ARG, attend(orow=252), "16 bytes")
    refused(L, ARG, attend(blocks=None), "go together")
    refused(L, ARG, attend(n=0), "go together")
    refused(L, ARG, attend(scale=float("nan")), "scale")
    refused(L, ARG, attend(scale=float("inf")), "scale")


@pytest.mark.parametrize("scale", [2.4e38, -2.4e38, 3.4e38, float("-inf")])
def test_a_scale_whose_power_of_two_is_infinite_is_refused(L, scale):
    """Scores are formed in powers of two, scale / ln 2 = 1.4427 scale: from 2.36e38 on that is no float."""
    refused(L, ARG, L.cerberus_paged_attention(pages(), table(), A, 256, A, 256, 2, 4, scale, None, 0, A, 1 << 30, None), "scale")


def test_workspace_follows_the_work_not_the_table(L):
    """A wide table or a large batch asks for no more partial results than the card has workgroups for."""
    pg = pages(n_kv_heads=8, head_dim=128, n_pages=1 << 20)
    small = L.cerberus_paged_workspace_bytes(pg, table(max_blocks=64, n_pages=1 << 20), 2, 32, 0)
    wide = L.cerberus_paged_workspace_bytes(pg, table(max_blocks=1 << 16, n_pages=1 << 20), 2, 32, 0)
    many = L.cerberus_paged_workspace_bytes(pg, table(max_seqs=1024, max_blocks=1 << 16, n_pages=1 << 20), 1024, 32, 0)
    assert 0 < small <= wide <= 64 << 20 and 0 < many <= 64 << 20


def test_step_arguments_without_a_context(L):
    pg, pt, st = pages(), table(), B.State()
    assert L.cerberus_paged_step(None, C.byref(st), pg, pt, 1, None, 0, A, 1 << 30, None) == ARG


def test_a_page_cache_needs_a_gpu():
    with pytest.raises(ValueError):
        B.PageCache(1, 8, 16, 2, 64, B.CERBERUS_BF16, 3, 4, device="cpu")


def test_constants_match_the_header():
    text = open(os.path.join(os.path.dirname(B.LIB_PATH), "..", "include", "cerberus.h")).read()
    for name, value in (("CERBERUS_DEV_BAD_PAGE", B.CERBERUS_DEV_BAD_PAGE), ("CERBERUS_MAX_SEQS", B.CERBERUS_MAX_SEQS)):
        assert f"{name} = {value}" in text
