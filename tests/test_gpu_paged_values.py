"""Infinite and NaN values in rows that the paged attention reads, and in rows it does not."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2410_13344_amd import binding as B
from tests.test_gpu_paged import check_attention, filled

BF16, F32 = B.CERBERUS_BF16, B.CERBERUS_F32


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lens", [[40, 19, 16], [1500, 700, 129]])     # whole, cut
def test_an_infinite_value_shows_in_its_column_alone(dtype, lens):
    """In the newest row, whose neighbours in the tile are read again in its place, and in one in the middle; the other columns
    and sequences are those of the finite cache, and rows that lie behind a sequence's end show nowhere."""
    c, k, v, table, q = filled(dtype, 4, 2, 64, 16, lens, seed=3)
    for value in (float("inf"), float("-inf"), float("nan")):
        bad = v.clone()
        for col, row in ((5, lens[0] - 1), (40, lens[0] // 2)):
            bad[table[0][row // 16], :, row % 16, col] = value
        c.v[0].copy_(bad)
        out = c.attention(0, q.cuda())
        assert not torch.isfinite(out[0, :, [5, 40]]).any()
        c.v[0].copy_(v)
        clean = c.attention(0, q.cuda())
        check_attention(clean, q, k, v, table, lens, 16, dtype)
        rest = [d for d in range(64) if d not in (5, 40)]
        assert torch.equal(out[0][:, rest], clean[0][:, rest]) and torch.equal(out[1:], clean[1:])
