"""Large batches whose sequences are cut, and choices over wide tables, against plain implementations in 64 bits."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2410_13344_amd import binding as B
from tests.test_gpu_paged import check_attention, filled, select_plain, with_bounds

BF16, F32 = B.CERBERUS_BF16, B.CERBERUS_F32


def mixed_lens(n, seed):
    """Empty, short and long sequences; the long ones, each cut into many pieces, spread over every 64 of them, two in a row at
    places that one lane looks after (64 apart) and at both ends."""
    rng = random.Random(seed)
    lens = [rng.choice([0, 1, 5, 16, 17, rng.randint(0, 40)]) for _ in range(n)]
    for b in {0, 1, 63, 64, 65, 129, 191, n // 2, n - 1}:
        if b < n:
            lens[b] = rng.randint(1100, 2600)
    return lens


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,heads,kv,dh", [(65, 6, 2, 128), (257, 2, 2, 64), (257, 17, 1, 64), (1024, 2, 1, 64)])
def test_attention_of_large_batches_that_are_cut(dtype, n, heads, kv, dh):
    lens = mixed_lens(n, n)
    c, k, v, table, q = filled(dtype, heads, kv, dh, 16, lens, seed=n)
    assert c.max_blocks * 16 > 1024                              # above that a launch cuts, whatever its size
    d = q.cuda()
    out = c.attention(0, d)
    check_attention(out, q, k, v, table, lens, 16, dtype)
    assert not out[[b for b, m in enumerate(lens) if m == 0]].any() and int(c.status) == 0
    assert torch.equal(c.attention(0, d), out)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_over_lists_of_a_large_batch_that_are_cut(dtype):
    """A list for each of 100 sequences, long enough to be cut, with empty places; 100 is below the number of lists that stay whole."""
    rng = random.Random(9)
    lens = mixed_lens(100, 3)
    c, k, v, table, q = filled(dtype, 4, 1, 64, 16, lens, seed=1)
    blocks = []
    for m in lens:
        held = -(-m // 16)
        row = rng.sample(range(held), min(held, rng.choice([0, 3, 45, 60])))
        blocks.append([row + [-1] * (60 - len(row))])
    out = c.attention(0, q.cuda(), blocks=torch.tensor(blocks, dtype=torch.int32, device="cuda"))
    check_attention(out, q, k, v, table, lens, 16, dtype, blocks=blocks)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dh", [64, 128])
def test_select_over_wide_tables(dtype, dh):
    """Tables of more than 1024 blocks: long lists and short ones, several key heads with queries of their own."""
    lens = [16 * 1300 + 5, 33, 16 * 1024, 16 * 1025, 0, 16 * 2047 + 5]
    c, bounds, table, q = with_bounds(dtype, 6, 3, dh, 16, lens, seed=dh)
    assert c.max_blocks > 1024
    d = q.cuda()
    for n in (1, 3, 64, 1025):
        assert torch.equal(c.select(0, d, n).cpu(), select_plain(q, bounds, table, lens, n, 16, 3)), n
