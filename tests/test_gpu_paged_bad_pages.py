"""Page numbers that no pool has, in tables and free lists: none becomes another page by its offset passing 32 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2410_13344_amd import binding as B
from paper_2410_13344_amd import synth
from tests import harness as H

BF16, F32 = B.CERBERUS_BF16, B.CERBERUS_F32


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def wrapping(page):
    """Page numbers whose rows, counted in 32 bits, are those of page 1 (and the usual ones outside a pool)."""
    around = 2 ** 32 // page
    return [v for v in (around + 1, 1 - around, 2 * around + 1, 1 - 2 * around) if -2 ** 31 <= v < 2 ** 31] + [-1, 6, 2 ** 31 - 1, -2 ** 31]


@pytest.mark.parametrize("rows", [2, 2500])                      # in one workgroup, in many
@pytest.mark.parametrize("page", [16, 64, 256])
def test_plan_gives_no_place_in_a_page_outside_the_pool(page, rows):
    for bad in wrapping(page):
        c = B.PageCache(0, 6, page, 1, 64, BF16, 3, 3)
        c.block_table.copy_(ints([[4, -1, -1], [bad, -1, -1], [-1, -1, -1]]))
        c.kv_len.copy_(ints([3, 5, 0]))
        c.free_pages[:2] = ints([2, bad])                       # the third sequence takes them from the end
        c.n_free.fill_(2)
        plan = c.plan(ints([1, 2, page + 1]), page + 4 + rows)
        want = [4 * page + 3, -1, -1] + [-1] * page + [2 * page] + [-1] * rows
        assert plan.slot.tolist() == want and int(c.status) == B.CERBERUS_DEV_BAD_PAGE, bad
        assert plan.row_start.tolist() == [0, 1, 3, page + 4] and plan.first_pos.tolist() == [3, 5, 0]
        assert c.kv_len.tolist() == [4, 7, page + 1] and int(c.n_free) == 0 and c.block_table[2].tolist() == [bad, 2, -1]


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_paged_step_writes_nothing_for_a_page_number_that_passes_32_bits(dtype):
    """Two sequences; the free list of the second one's new page names page 1 in 32 bits, which is the first one's."""
    pair = H.Pair("tiny", dtype, "tiny", seed=0, max_batch=2, kv_capacity=192)
    eng, cfg = pair.engine, pair.cfg
    for bad in wrapping(16):
        sp = eng.new_state()
        for b, n in enumerate((20, 16)):
            eng.prefill(sp, 2, b, synth.make_token_ids(n, cfg["vocab"], seed=b).to(torch.int32).cuda())
        cache = B.PageCache(cfg["n_layers"], 6, 16, cfg["n_heads"], cfg["head_dim"], dtype, 2, 3)
        eng.move_prompts(sp, cache, [20, 16])
        assert cache.block_table[0, :2].tolist() == [0, 1]
        kept = cache.k.clone(), cache.v.clone(), cache.bounds.clone()
        cache.free_pages.fill_(bad)
        eng.paged_step(sp, cache, 2)
        assert int(cache.status) == B.CERBERUS_DEV_BAD_PAGE, bad
        for now, before in zip((cache.k, cache.v), kept):
            assert (now[:, 1, :, 4] != before[:, 1, :, 4]).any()                            # the first one's row
            now[:, 1, :, 4] = before[:, 1, :, 4]
            assert torch.equal(now, before), bad
        assert torch.equal(cache.bounds, kept[2])
    eng.close()


# ------------------------------------------------------------------------------------------------
# the choice of blocks
# ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("blocks", [12, 1500])                   # scored and picked in one launch, in two
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_select_takes_blocks_outside_the_pool_after_all_others(dtype, blocks):
    """Scores below zero, one of -inf, one a tie: every block of a page that is there goes before those of pages that are not; the
    newest and the first go by their places."""
    page, dh, held = 16, 64, 12
    c = B.PageCache(1, held, page, 2, dh, dtype, 2, blocks)
    c.block_table[:, :held] = torch.arange(held, dtype=torch.int32, device="cuda")
    c.block_table[1, 0] = held                                   # the first one's page is not there either
    for b in range(2):
        c.block_table[b, 4], c.block_table[b, 7], c.block_table[b, 9] = held, -3, 2 ** 31 - 1
    c.kv_len.fill_(held * page - 5)
    for j in range(held):                                        # block j scores -(j % 4 + 1) * 64 * 4, block 5 -inf
        c.bounds[0, j] = -(j % 4 + 1.0)
    c.bounds[0, 5] = float("-inf")
    q = torch.ones(2, 8, dh, dtype=c.dtype, device="cuda")       # groups of four queries
    there = [8, 1, 2, 6, 10, 3, 5]                               # by score, then place; 0 and 11 go first
    for n in range(1, held + 1):
        got = c.select(0, q, n).cpu()
        best = ([11, 0] + there + [4, 7, 9])[:n]
        want = torch.tensor(sorted(best), dtype=torch.int32).expand(2, 2, n)
        assert torch.equal(got, want), (n, got.tolist())


def test_select_among_nothing_but_pages_outside_the_pool():
    for blocks in (9, 1100):
        c = B.PageCache(1, 4, 16, 1, 64, BF16, 1, blocks)
        c.block_table.fill_(77)
        c.kv_len.fill_(9 * 16)
        q = torch.ones(1, 1, 64, dtype=c.dtype, device="cuda")
        for n in (1, 2, 5, 8, 9):
            assert c.select(0, q, n)[0, 0].tolist() == ([8] if n == 1 else list(range(n - 1)) + [8])
