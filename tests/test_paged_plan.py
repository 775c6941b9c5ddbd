"""How the paged attention's rows are cut, on the CPU: the kernel's rule, written out here, against the number of workgroups and the
room for partial results that the host gives a launch."""
import ctypes as C
import random

import pytest

from paper_2410_13344_amd import binding as B

TARGET, TURNS = 2048, 4


def items(batch, most, unit, per_head):
    f = getattr(B.lib(), "_ZN4cerb21paged_attention_itemsEixii")         # int paged_attention_items(int, long long, int, int)
    f.restype, f.argtypes = C.c_int, [C.c_int, C.c_longlong, C.c_int, C.c_int]
    return f(batch, most, unit, per_head)


def room(n_heads, n_kv_heads, head_dim):
    """Partial results (of all heads) that the workspace holds."""
    f = getattr(B.lib(), "_ZN4cerb21paged_attention_bytesEiii")
    f.restype, f.argtypes = C.c_size_t, [C.c_int] * 3
    return f(n_heads, n_kv_heads, head_dim) // (n_heads * (head_dim + 2) * 4)


def piece(lens, unit, per_head):
    total, half, quarter = sum(lens), (per_head + 1) // 2, (per_head + 3) // 4
    rows = max(-(-total // per_head), min(-(-total // half), 1024), min(-(-total // quarter), 512), 1)
    return min(-(-rows // unit) * unit, 2 ** 31 - 1)


@pytest.mark.parametrize("heads,kv", [(32, 32), (32, 8), (40, 40), (1, 1), (16, 1), (24, 1), (64, 8), (4096, 1024), (65535, 1), (65535, 3)])
@pytest.mark.parametrize("unit", [64, 128])
def test_every_piece_has_a_workgroup_and_room_for_its_partial_result(heads, kv, unit):
    rng = random.Random(heads * 131 + kv)
    tiles = (heads // kv + 15) // 16
    per_head = max(1, TARGET // (kv * tiles))
    slots = room(heads, kv, 128)
    for i in range(400):
        batch = rng.choice([1, 1, 2, 3, 16, 64, 1024])
        most = rng.choice([TURNS * unit + 16, 1040, 4096, 131072, 2 ** 31 - 256])
        lens = [rng.choice([0, 1, most, rng.randint(0, most), rng.randint(0, min(most, 3000))]) for _ in range(batch)]
        if i % 4 == 0:
            lens = [most] * batch
        p = piece(lens, unit, per_head)
        pieces = [max(1, -(-n // p)) for n in lens]
        assert sum(pieces) <= items(batch, most, unit, per_head), (batch, most, i)
        assert sum(n for n in pieces if n > 1) <= slots, (batch, most, i)
        assert sum(pieces) < 1 << 16 and sum(n for n in pieces if n > 1) < 1 << 15    # the kernel scans both in one word
