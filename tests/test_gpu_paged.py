"""The cache in pages on an MI355X against plain implementations in 64 bits: plan, store, choice of blocks, attention of one
token, and the step that calls them all."""
import math
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2410_13344_amd import binding as B
from paper_2410_13344_amd import synth
from tests import harness as H

BF16, F32 = B.CERBERUS_BF16, B.CERBERUS_F32


# ------------------------------------------------------------------------------------------------
# plain implementations
# ------------------------------------------------------------------------------------------------

def plan_plain(state, new, max_rows, page, blocks):
    """One sequence after the other: first the ends, then first come, first served."""
    lens, table, free = list(state["lens"]), [list(r) for r in state["table"]], list(state["free"])
    cap, status = blocks * page, 0
    for b, m in enumerate(new):
        if m < 0:
            if 0 <= lens[b] <= cap:
                free += table[b][:-(-lens[b] // page)]
            lens[b] = 0
    row_start, first, slot, wanted, had = [0], [], [-1] * max_rows, 0, len(free)
    for b, m in enumerate(new):
        start = row_start[-1]
        row_start.append(min(start + max(m, 0), 2 ** 31 - 1))           # (the largest an int32 holds)
        if m < 0:
            first.append(-1)
            continue
        ok = 0 <= lens[b] <= cap and lens[b] + m <= cap and start + m <= max_rows
        need = -(-(lens[b] + m) // page) - -(-lens[b] // page) if ok else 0
        wanted += need
        if not ok or (need and wanted > had):
            first.append(-1)
            status |= B.CERBERUS_DEV_KV_OVERFLOW
            continue
        for j in range(need):
            table[b][-(-lens[b] // page) + j] = free.pop()
        first.append(lens[b])
        for i in range(m):
            pos = lens[b] + i
            slot[start + i] = table[b][pos // page] * page + pos % page
        lens[b] += m
    return {"lens": lens, "table": table, "free": free}, row_start, first, slot, status


def attend_plain(q, k, v, table, lens, scale, page, blocks=None):
    """(out, sum of p |v|, largest sum of |q k| scale) per sequence and head in 64 bits; q [b][heads][dh], pools [pages][kv][page][dh]."""
    n, heads, dh = q.shape
    kv = k.shape[1]
    out, mass, peak = torch.zeros(n, heads, dh, dtype=torch.float64), torch.zeros(n, heads, dh, dtype=torch.float64), torch.zeros(n, heads, 1, dtype=torch.float64)
    for b in range(n):
        L = lens[b]
        for h in range(heads):
            hk = h // (heads // kv)
            if blocks is None:
                rows = list(range(L))
            else:
                rows = [j * page + i for j in blocks[b][hk] if 0 <= j < -(-L // page) for i in range(page) if j * page + i < L]
            if not rows:
                continue
            r = torch.tensor(rows)
            p = torch.tensor(table[b])[r // page]
            kk, vv = k[p, hk, r % page].double(), v[p, hk, r % page].double()
            s = (kk * q[b, h].double()).sum(1) * scale
            w = torch.softmax(s, 0)
            out[b, h] = (w[:, None] * vv).sum(0)
            mass[b, h] = (w[:, None] * vv.abs()).sum(0)
            peak[b, h] = ((kk * q[b, h].double()).abs().sum(1) * abs(scale)).max()
    return out, mass, peak


def attend_bound(want, mass, peak, rows, dh, dtype):
    """How far the kernel may be off: the output's rounding, half a step; and on every probability-weighted value a relative
    error of the score (dh products and sums, the scale and the base change of the exponential in 24 bits, of a
    sum whose terms add up to `peak`; it enters numerator and denominator), of the exponential itself and of the sums over
    the rows.  bf16 mode multiplies values by probabilities in two bf16 planes, 2^-17 relative, once."""
    eps = 2.0 ** -24
    half_step = 2.0 ** -8 if dtype == BF16 else eps
    rel = 2 * eps * ((dh + 8) * peak + 8 + rows) + (2.0 ** -16 if dtype == BF16 else 0.0)
    return half_step * (want.abs() + rel * mass) + rel * mass + 1e-30


def select_plain(q, bounds, table, lens, n_select, page, kv):
    n, heads, dh = q.shape
    out = torch.full((n, kv, n_select), -1, dtype=torch.int32)
    for b in range(n):
        held = -(-lens[b] // page)
        for h in range(kv):
            total = q[b, h * (heads // kv):(h + 1) * (heads // kv)].double().sum(0)
            score = []
            for j in range(held):
                lo, hi = bounds[table[b][j], h, 0].double(), bounds[table[b][j], h, 1].double()
                s = float((total * torch.where(total >= 0, hi, lo)).sum())
                score.append(math.inf if math.isnan(s) else s)
            order = sorted(range(held), key=lambda j: (-(j == held - 1), -(j == 0), -score[j], j))
            pick = sorted(order[:n_select])
            out[b, h, :len(pick)] = torch.tensor(pick, dtype=torch.int32)
    return out


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------

def filled(dtype, heads, kv, dh, page, lens, seed=0, spare=3, poison=True, extra_blocks=0):
    """A cache whose sequences hold `lens` rows, pages in random order; everything that no sequence holds is NaN."""
    rng = random.Random(seed)
    held = [-(-v // page) for v in lens]
    n_pages, blocks = sum(held) + spare, max(held + [1]) + extra_blocks
    c = B.PageCache(1, n_pages, page, kv, dh, dtype, len(lens), blocks)
    g = torch.Generator().manual_seed(seed)
    shape = (n_pages, kv, page, dh)
    k, v = torch.randn(shape, generator=g).to(c.dtype), torch.randn(shape, generator=g).to(c.dtype)
    order = list(range(n_pages))
    rng.shuffle(order)
    table = [[order.pop() for _ in range(m)] + [-7] * (blocks - m) for m in held]
    if poison:
        live = torch.zeros(n_pages, page, dtype=torch.bool)
        for b, length in enumerate(lens):
            for r in range(length):
                live[table[b][r // page], r % page] = True
        dead = ~live[:, None, :, None].expand(shape)
        k[dead], v[dead] = float("nan"), float("nan")
        k[:, :, -1:][dead[:, :, -1:]] = float("inf")
    c.k[0].copy_(k)
    c.v[0].copy_(v)
    c.block_table.copy_(torch.tensor(table, dtype=torch.int32))
    c.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
    c.free_pages[:len(order)] = torch.tensor(order, dtype=torch.int32, device="cuda")
    c.n_free.fill_(len(order))
    q = torch.randn(len(lens), heads, dh, generator=g).to(c.dtype)
    return c, k, v, table, q


def check_attention(got, q, k, v, table, lens, page, dtype, scale=None, blocks=None):
    scale = q.shape[2] ** -0.5 if scale is None else scale
    want, mass, peak = attend_plain(q, k, v, table, lens, scale, page, blocks)
    rows = max(lens) if blocks is None else page * len(blocks[0][0])
    off = (got.double().cpu() - want).abs()
    tol = attend_bound(want, mass, peak, rows, q.shape[2], dtype)
    assert torch.isfinite(got).all()
    assert (off <= tol).all(), (float((off - tol).max()), float(off.max()))


# ------------------------------------------------------------------------------------------------
# plan
# ------------------------------------------------------------------------------------------------

def run_plan(page, blocks, n_pages, lens, new, max_rows=None, seed=0, free=None):
    rng = random.Random(seed)
    held = [-(-max(0, min(v, blocks * page)) // page) if 0 <= v <= blocks * page else 0 for v in lens]
    c = B.PageCache(0, n_pages, page, 1, 64, BF16, len(lens), blocks)
    order = list(range(n_pages))
    rng.shuffle(order)
    table = [[order.pop() for _ in range(m)] + [-5] * (blocks - m) for m in held]
    free = order if free is None else order[:free]
    state = {"lens": lens, "table": table, "free": free}
    c.block_table.copy_(torch.tensor(table, dtype=torch.int32))
    c.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
    c.free_pages.fill_(-9)
    c.free_pages[:len(free)] = torch.tensor(free, dtype=torch.int32, device="cuda")
    c.n_free.fill_(len(free))
    max_rows = sum(max(m, 0) for m in new) if max_rows is None else max_rows
    plan = c.plan(torch.tensor(new, dtype=torch.int32, device="cuda"), max_rows)
    n = len(new)
    after, row_start, first, slot, status = plan_plain(state, new, max_rows, page, blocks)
    assert int(c.n_free) == len(after["free"])
    assert c.free_pages[:len(after["free"])].tolist() == after["free"]
    assert c.kv_len.tolist() == after["lens"]
    assert c.block_table.tolist() == after["table"]
    assert plan.row_start.tolist() == row_start and plan.first_pos.tolist() == first
    assert plan.slot[:max_rows].tolist() == slot
    assert int(c.status) == status
    return c, first


@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 257, 1024])
def test_plan_of_a_mixed_batch(page, n):
    rng = random.Random(n * 1000 + page)
    lens = [rng.choice([0, 1, page - 1, page, page + 1, rng.randint(0, 5 * page)]) for _ in range(n)]
    new = [rng.choice([1, 1, 0, -1, -5, page, rng.randint(0, 4 * page)]) for _ in range(n)]
    pages = sum(-(-v // page) for v in lens)
    run_plan(page, 12, pages + 8 * n + 4, lens, new, seed=n)
    run_plan(page, 12, pages + n, lens, new, seed=n)           # short of pages somewhere along the batch


def test_plan_of_long_prompts_and_rows_beyond_one_workgroup():
    run_plan(16, 1024, 2600, [0, 16000, 5, 0], [16384, 384, 9000, 1])
    run_plan(16, 300, 1000, [0] * 3, [1365, 1365, 1366])       # 4096 rows
    run_plan(16, 300, 1000, [0] * 3, [1365, 1366, 1366])


def test_plan_refusals():
    _, first = run_plan(16, 4, 40, [60, 64, 1, 0], [5, 1, 63, 65])             # the table has room for 64 rows
    assert first == [-1, -1, 1, -1]
    _, first = run_plan(16, 4, 40, [0, 0, 0], [20, 30, 10], max_rows=50)       # the slot map for 50
    assert first == [0, 0, -1]
    _, first = run_plan(16, 8, 5, [0, 15, 0, 3], [64, 1, 17, 1])               # 2 pages free: who needs none still runs
    assert first == [-1, 15, -1, 3]
    _, first = run_plan(16, 8, 3, [30, 0], [-1, 32])                           # pages of one that ends serve the next
    assert first == [-1, 0]
    _, first = run_plan(16, 4, 10, [-3, 65, 2 ** 31 - 1, 7], [1, 0, -1, 1])    # lengths that no table holds
    assert first == [-1, -1, -1, 7]
    _, first = run_plan(16, 4, 10, [0, 0, 3], [2 ** 31 - 1, 2 ** 31 - 1, 1], max_rows=4)
    assert first == [-1, -1, -1]
    run_plan(16, 4, 10, [5, 6], [0, 0], max_rows=0)


def test_plan_leaves_other_sequences_and_repeats():
    """Plans of a part of the table, grown token by token and ended, come back to where they began."""
    c = B.PageCache(0, 20, 16, 1, 64, BF16, 6, 5)
    start = c.words.clone()
    one = torch.ones(4, dtype=torch.int32, device="cuda")
    c.kv_len[5] = 33
    seen = []
    for _ in range(40):
        p = c.plan(one, 4)
        seen.append(p.slot.tolist())
    assert c.kv_len.tolist() == [40, 40, 40, 40, 0, 33] and int(c.n_free) == 20 - 12
    flat = [s for r in seen for s in r]
    assert len(set(flat)) == len(flat) and min(flat) >= 0 and max(flat) < 20 * 16
    c.plan(-one, 0)
    assert int(c.n_free) == 20 and sorted(c.free_pages.tolist()) == list(range(20)) and int(c.status) == 0
    assert c.kv_len.tolist() == [0, 0, 0, 0, 0, 33]
    assert start.numel() == c.words.numel()


# ------------------------------------------------------------------------------------------------
# store
# ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,kv,dh", [(BF16, 1, 128), (BF16, 5, 64), (F32, 3, 128), (F32, 2, 64)])
@pytest.mark.parametrize("page", [16, 32, 256])
def test_store_of_ragged_rows_and_bounds(dtype, kv, dh, page):
    lens, new = [0, 1, page - 1, page, 0, 2 * page + 3, 7], [1, 1, 1, 1, 3 * page + 1, page, 0]
    g = torch.Generator().manual_seed(page)
    c = B.PageCache(2, 40, page, kv, dh, dtype, len(lens), 8)
    n0, n1 = sum(lens), sum(new)
    p0 = c.plan(torch.tensor(lens, dtype=torch.int32, device="cuda"), n0)
    rows = torch.randn(n0, 2, kv, dh, generator=g).to(c.dtype)
    dev = rows.cuda()
    c.store(1, dev[:, 0], dev[:, 1], p0.slot)
    p1 = c.plan(torch.tensor(new, dtype=torch.int32, device="cuda"), n1 + 5)       # (slots behind the last row are -1)
    more = torch.randn(n1 + 5, 2, kv, dh, generator=g).to(c.dtype)
    heads_first = more.permute(1, 2, 0, 3).contiguous().cuda()                     # [K,V][kv][rows][dh]
    c.store(1, heads_first[0].transpose(0, 1), heads_first[1].transpose(0, 1), p1.slot)
    want_k, want_v = torch.zeros_like(c.k[1].cpu()), torch.zeros_like(c.v[1].cpu())
    fill = {}
    for plan, data in ((p0, rows), (p1, more)):
        for i, s in enumerate(plan.slot.tolist()):
            if s >= 0:
                want_k[s // page, :, s % page], want_v[s // page, :, s % page] = data[i, 0], data[i, 1]
                fill[s // page] = max(fill.get(s // page, 0), s % page + 1)
    assert torch.equal(c.k[1].cpu(), want_k) and torch.equal(c.v[1].cpu(), want_v)
    bounds = c.bounds[1].cpu()
    for p in range(40):
        n = fill.get(p, 0)
        want = torch.stack([want_k[p, :, :n].amin(1), want_k[p, :, :n].amax(1)], 1) if n else torch.zeros(kv, 2, dh, dtype=c.dtype)
        assert torch.equal(bounds[p], want), p
    assert not c.k[0].any() and not c.bounds[0].any() and int(c.status) == 0       # the other layer


def test_store_skips_and_reports_rows_without_a_place():
    c = B.PageCache(1, 4, 16, 2, 64, F32, 1, 4)
    rows = torch.arange(5 * 2 * 64, dtype=torch.float32, device="cuda").view(5, 2, 64)
    slot = torch.tensor([-1, 3, -2 ** 31, 4 * 16 - 1, -1], dtype=torch.int32, device="cuda")
    c.store(0, rows, rows, slot)
    assert int(c.status) == 0
    want = torch.zeros(4, 2, 16, 64)
    want[0, :, 3], want[3, :, 15] = rows[1].cpu(), rows[3].cpu()
    assert torch.equal(c.k[0].cpu(), want) and torch.equal(c.v[0].cpu(), want)
    c.store(0, rows[:2], rows[:2], torch.tensor([64, 2 ** 31 - 1], dtype=torch.int32, device="cuda"))
    assert torch.equal(c.k[0].cpu(), want) and int(c.status) == B.CERBERUS_DEV_BAD_PAGE


def test_store_bounds_keep_nan_and_infinities():
    c = B.PageCache(1, 2, 16, 1, 64, BF16, 1, 2)
    rows = torch.zeros(3, 1, 64, dtype=torch.bfloat16)
    rows[0, 0, 0], rows[1, 0, 1], rows[2, 0, 2], rows[:, 0, 3] = float("nan"), float("inf"), float("-inf"), -2.5
    d = rows.cuda()
    c.store(0, d[:2], d[:2], torch.tensor([0, 1], dtype=torch.int32, device="cuda"))
    c.store(0, d[2:], d[2:], torch.tensor([2], dtype=torch.int32, device="cuda"))
    lo, hi = c.bounds[0, 0, 0, 0].float().cpu(), c.bounds[0, 0, 0, 1].float().cpu()
    assert lo[0].isnan() and hi[0].isnan() and hi[1] == float("inf") and lo[1] == 0 and lo[2] == float("-inf") and hi[2] == 0
    assert lo[3] == hi[3] == -2.5


def test_store_of_many_rows():
    """More rows than workgroups, runs that cross any chunk of rows."""
    for n, page in ((5000, 16), (5000, 256)):
        c = B.PageCache(1, 400, page, 4, 64, BF16, 3, 400)
        new = [n - 1501, 1500, 1]
        p = c.plan(torch.tensor(new, dtype=torch.int32, device="cuda"), n)
        rows = torch.randn(n, 4, 64, device="cuda").to(torch.bfloat16)
        c.store(0, rows, rows, p.slot)
        s = p.slot.long()
        assert torch.equal(c.k[0][s // page, :, s % page], rows) and torch.equal(c.v[0][s // page, :, s % page], rows)
        full = c.block_table[0, :new[0] // page].long()
        assert torch.equal(c.bounds[0][full, :, 0], c.k[0][full].amin(2)) and torch.equal(c.bounds[0][full, :, 1], c.k[0][full].amax(2))
        last = int(c.block_table[2, 0])
        assert torch.equal(c.bounds[0][last, :, 0], rows[-1]) and torch.equal(c.bounds[0][last, :, 1], rows[-1])


# ------------------------------------------------------------------------------------------------
# attention
# ------------------------------------------------------------------------------------------------

LENS = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 300, 511, 513, 700]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads,kv,dh,page", [(4, 4, 64, 16), (4, 4, 128, 16), (8, 2, 128, 32), (5, 1, 64, 64), (16, 1, 128, 256),
                                             (17, 1, 64, 16), (40, 2, 128, 16), (33, 1, 128, 128), (14, 2, 64, 256)])
def test_attention_over_ragged_lengths(dtype, heads, kv, dh, page):
    c, k, v, table, q = filled(dtype, heads, kv, dh, page, LENS, seed=heads)
    out = c.attention(0, q.cuda())
    check_attention(out, q, k, v, table, LENS, page, dtype)
    assert not out[0].any() and int(c.status) == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lens", [[1], [40], [1025], [5000], [3000, 2], [0], [0, 0, 0], [2100] * 3])
def test_attention_of_few_sequences(dtype, lens):
    """Few rows and long ones are cut along the length and joined; short ones are not."""
    c, k, v, table, q = filled(dtype, 4, 2, 128, 16, lens, seed=len(lens), extra_blocks=9)
    check_attention(c.attention(0, q.cuda()), q, k, v, table, lens, 16, dtype)


def test_attention_of_the_largest_batch():
    lens = [(7 * i) % 70 for i in range(1024)]
    c, k, v, table, q = filled(BF16, 2, 1, 64, 16, lens, poison=False)
    check_attention(c.attention(0, q.cuda()), q, k, v, table, lens, 16, BF16)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_far_scores(dtype):
    """Scores hundreds apart, in rising, falling and single-peak order along the cache, and equal ones; an own scale."""
    lens, page, dh = [400, 400, 400, 400], 16, 64
    c, k, v, table, q = filled(dtype, 2, 1, dh, page, lens, poison=False)
    q[:] = 1.0
    ramp = torch.arange(400.0) / 8
    for b, values in enumerate([ramp, ramp.flip(0), 50 - (ramp - 25).abs() * 4, torch.zeros(400)]):
        for r in range(400):
            k[table[b][r // page], 0, r % page] = values[r].to(k.dtype)
    c.k[0].copy_(k)
    check_attention(c.attention(0, q.cuda(), scale=0.25), q, k, v, table, lens, page, dtype, scale=0.25)
    check_attention(c.attention(0, q.cuda(), scale=-0.125), q, k, v, table, lens, page, dtype, scale=-0.125)
    check_attention(c.attention(0, q.cuda(), scale=0.0), q, k, v, table, lens, page, dtype, scale=0.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_passes_on_infinities_of_rows_it_reads(dtype):
    """A key of -inf scores takes a row out; a sequence of nothing but such rows gives zeros; a NaN in a row that is read shows."""
    c, k, v, table, q = filled(dtype, 2, 1, 64, 16, [40, 40, 40], poison=False)
    q[:] = 1.0
    k[table[0][0], 0, :16] = float("-inf")
    for j in range(3):
        k[table[1][j]] = float("-inf")
    v[table[2][1], 0, 3, 5] = float("nan")
    c.k[0].copy_(k)
    c.v[0].copy_(v)
    out = c.attention(0, q.cuda()).double().cpu()
    ref, mass, peak = attend_plain(q[:1], torch.nan_to_num(k, neginf=-1e4), v, table[:1], [40], 0.125, 16)
    assert (out[0] - ref[0]).abs().max() < 2.0 ** -7 * mass.max() and not out[1].any()
    assert out[2, :, 5].isnan().all() and torch.isfinite(out[2, :, :5]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("page", [16, 64, 128])
def test_attention_over_chosen_blocks(dtype, page):
    """In any order, with holes, doubles, indexes past the length, none at all, and the block that is not full."""
    lens = [5 * page + 7, 3 * page, 9 * page + 1, 0, 20]
    c, k, v, table, q = filled(dtype, 6, 2, 128, page, lens, seed=page)
    blocks = [[[5, 0, 3, -1], [1, 2, -1, -1]], [[-1, -1, -1, -1], [2, 7, 0, 3]], [[9, 8, 1, 0], [4, -1, 4, 9]],
              [[0, 1, -1, -1], [-1] * 4], [[0, 1, 2, 3], [3, 2, 1, -2 ** 31]]]
    out = c.attention(0, q.cuda(), blocks=torch.tensor(blocks, dtype=torch.int32, device="cuda"))
    check_attention(out, q, k, v, table, lens, page, dtype, blocks=blocks)
    assert not out[1, :3].any() and not out[3].any() and int(c.status) == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_over_many_chosen_blocks(dtype):
    rng = random.Random(4)
    lens = [4000, 4000 - 33]
    c, k, v, table, q = filled(dtype, 8, 2, 64, 16, lens)
    blocks = [[sorted(rng.sample(range(250), 180)) for _ in range(2)] for _ in range(2)]
    out = c.attention(0, q.cuda(), blocks=torch.tensor(blocks, dtype=torch.int32, device="cuda"))
    check_attention(out, q, k, v, table, lens, 16, dtype, blocks=blocks)


def test_attention_counts_what_the_tables_hold():
    """Page numbers outside the pool are no rows, a length above the table's room is that room, below zero none."""
    lens = [40, 64, 9]
    c, k, v, table, q = filled(BF16, 2, 1, 64, 16, lens)
    c.kv_len.copy_(torch.tensor([40, 2 ** 31 - 1, -4], dtype=torch.int32))
    out = c.attention(0, q.cuda())
    check_attention(out[:2], q[:2], k, v, table[:2], lens[:2], 16, BF16)
    assert not out[2].any() and int(c.status) == 0
    c.block_table[0, 1] = c.n_pages
    c.block_table[1, 0] = -1
    out = c.attention(0, q.cuda())
    assert int(c.status) == B.CERBERUS_DEV_BAD_PAGE
    check_attention(out[:2], q[:2], k, v, table[:2], lens[:2], 16, BF16, blocks=[[[0, 2, -1]], [[1, 2, 3]]])


def test_attention_strided_rows_and_given_outputs():
    lens = [33, 70]
    for dtype in (BF16, F32):
        c, k, v, table, q = filled(dtype, 4, 2, 64, 16, lens)
        wide = torch.full((2, 12, 64), 7.0, dtype=c.dtype, device="cuda")          # q as a slice of a projection's output
        wide[:, 4:8] = q.cuda()
        out = torch.full((2, 9, 64), 3.0, dtype=c.dtype, device="cuda")
        got = c.attention(0, wide[:, 4:8], out=out[:, 1:5])
        check_attention(got, q, k, v, table, lens, 16, dtype)
        assert (out[:, 0] == 3).all() and (out[:, 5:] == 3).all()
        one = wide[:1, 4:8].expand(2, 4, 64)                                       # one query for all sequences
        check_attention(c.attention(0, one), q[:1].expand(2, 4, 64), k, v, table, lens, 16, dtype)


def test_attention_past_32_bits_of_offset():
    """Pages whose elements lie more than 2^32 bytes and more than 2^31 elements into the pool."""
    c = B.PageCache(1, 140000, 16, 8, 128, BF16, 2, 4)                              # 2.3e9 elements, 4.6 GB each of K and V
    lens, table = [40, 35], [[139999, 131072, 139001], [5, 138000, 4]]
    g = torch.Generator().manual_seed(3)
    small, at = [], {}
    for row in table:
        small.append([at.setdefault(p, len(at)) for p in row])
    k, v = torch.randn(6, 8, 16, 128, generator=g).bfloat16(), torch.randn(6, 8, 16, 128, generator=g).bfloat16()
    rows_k, rows_v, slots = [], [], []
    for b, n in enumerate(lens):
        for r in range(n):
            rows_k.append(k[small[b][r // 16], :, r % 16])
            rows_v.append(v[small[b][r // 16], :, r % 16])
            slots.append(table[b][r // 16] * 16 + r % 16)
    c.store(0, torch.stack(rows_k).cuda(), torch.stack(rows_v).cuda(), torch.tensor(slots, dtype=torch.int32, device="cuda"))
    c.block_table[:, :3] = torch.tensor(table, dtype=torch.int32, device="cuda")
    c.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
    q = torch.randn(2, 8, 128, generator=g).bfloat16()
    check_attention(c.attention(0, q.cuda()), q, k, v, small, lens, 16, BF16)
    assert torch.equal(c.bounds[0, 139999, :, 0].cpu(), k[at[139999]].amin(1))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_of_many_heads_and_key_heads(dtype):
    """Head layouts that leave the last group of eight workgroups, or of sixteen queries, part empty."""
    lens = [700, 33, 0, 129]
    for heads, kv in ((1, 1), (3, 3), (9, 9), (35, 1), (66, 2), (51, 3), (70, 7)):
        c, k, v, table, q = filled(dtype, heads, kv, 64, 16, lens, seed=heads)
        check_attention(c.attention(0, q.cuda()), q, k, v, table, lens, 16, dtype)


def test_attention_gives_the_same_bits_again():
    c, k, v, table, q = filled(BF16, 8, 2, 128, 16, [4000, 17, 900])
    d = q.cuda()
    first = c.attention(0, d)
    for _ in range(5):
        assert torch.equal(c.attention(0, d), first)


# ------------------------------------------------------------------------------------------------
# choice of blocks
# ------------------------------------------------------------------------------------------------

def with_bounds(dtype, heads, kv, dh, page, lens, seed=0):
    c, k, v, table, q = filled(dtype, heads, kv, dh, page, lens, seed=seed, poison=False)
    g = torch.Generator().manual_seed(seed + 1)
    mid = torch.randn(c.n_pages, kv, 1, dh, generator=g)
    half = torch.rand(c.n_pages, kv, 1, dh, generator=g)
    bounds = torch.cat([mid - half, mid + half], 2).to(c.dtype)
    c.bounds[0].copy_(bounds)
    return c, bounds, table, q


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads,kv,dh,page", [(4, 4, 64, 16), (8, 2, 128, 16), (24, 1, 128, 32), (6, 3, 64, 64)])
@pytest.mark.parametrize("n_select", [1, 2, 3, 7, 40, 100])
def test_select(dtype, heads, kv, dh, page, n_select):
    lens = [0, 1, page, page + 1, 2 * page, 7 * page + 3, 40 * page, 41 * page - 1, 100 * page]
    c, bounds, table, q = with_bounds(dtype, heads, kv, dh, page, lens, seed=n_select)
    got = c.select(0, q.cuda(), n_select).cpu()
    assert torch.equal(got, select_plain(q, bounds, table, lens, n_select, page, kv))


def test_select_among_many_blocks():
    lens = [16 * 5000, 16 * 1024, 16 * 1025 + 1, 16 * 2047 + 5]
    c, bounds, table, q = with_bounds(BF16, 2, 1, 64, 16, lens)
    for n in (1, 2, 64, 1000, 4999):
        assert torch.equal(c.select(0, q.cuda(), n).cpu(), select_plain(q, bounds, table, lens, n, 16, 1)), n


def test_select_ties_nan_and_infinities():
    lens = [16 * 50, 16 * 50, 16 * 50, 16 * 50]
    for dtype in (BF16, F32):
        c, bounds, table, q = with_bounds(dtype, 2, 1, 64, 16, lens)
        for j in range(50):
            bounds[table[0][j]] = 0.5                                              # all alike: the lowest indexes
            bounds[table[1][j]] = [1.0, 2.0, 3.0][j % 3]                           # a tie at the border
        q[0], q[1] = 1.0, 1.0
        bounds[table[2][30], 0, :, 7] = float("nan")                               # counts as the highest
        bounds[table[2][20], 0, 1] = float("inf")
        bounds[table[2][20], 0, 0] = float("-inf")
        bounds[table[2][25], 0] = float("-inf")
        q[2, :, 0] = 0.0
        q[3] = -0.0                                                                # zeros of either sign are one score
        bounds[table[3][::2]] *= -1
        c.bounds[0].copy_(bounds)
        for n in (1, 2, 3, 4, 5, 20, 49, 50):
            got = c.select(0, q.cuda(), n).cpu()
            assert torch.equal(got, select_plain(q, bounds, table, lens, n, 16, 1)), n


def test_select_leaves_out_pages_outside_the_pool_last():
    """A page number outside the pool scores nothing and reads nothing; the attention reports it."""
    c, bounds, table, q = with_bounds(BF16, 2, 1, 64, 16, [160])
    c.block_table[0, 4] = 10 ** 6
    got = c.select(0, q.cuda(), 10).cpu()
    assert got[0, 0].tolist() == list(range(10))


# ------------------------------------------------------------------------------------------------
# together, as a server uses them
# ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_server_loop(dtype):
    """Prompts come, tokens are added, sequences end and others take their pages, over layers and with blocks chosen; every
    turn's attention against 64 bits over a copy of the rows that the host keeps."""
    page, kv, heads, dh, layers = 16, 2, 6, 64, 2
    rng = random.Random(1)
    g = torch.Generator().manual_seed(2)
    c = B.PageCache(layers, 60, page, kv, dh, dtype, 5, 12)
    rows = [[torch.zeros(2, 0, kv, dh, dtype=c.dtype) for _ in range(5)] for _ in range(layers)]   # [K,V][n][kv][dh]
    lens = [0] * 5
    for turn in range(12):
        new = [rng.choice([1, 1, 1, 30, -1]) if lens[b] else rng.choice([5, 33, 100, 0]) for b in range(5)]
        new = [m if lens[b] + m <= 12 * page else -1 for b, m in enumerate(new)]
        n = sum(max(m, 0) for m in new)
        plan = c.plan(torch.tensor(new, dtype=torch.int32, device="cuda"), n + 3)
        lens = [0 if m < 0 else l + m for l, m in zip(lens, new)]
        assert c.kv_len.tolist() == lens and int(c.status) == 0
        for l in range(layers):
            data = torch.randn(n + 3, 3, kv, dh, generator=g).to(c.dtype)
            dev = data.cuda()
            c.store(l, dev[:, 0], dev[:, 1], plan.slot)
            at = 0
            for b, m in enumerate(new):
                if m < 0:
                    rows[l][b] = rows[l][b][:, :0]
                else:
                    rows[l][b] = torch.cat([rows[l][b], data[at:at + m, :2].transpose(0, 1)], 1)
                    at += m
            q = torch.randn(5, heads, dh, generator=g).to(c.dtype)
            pool_k, pool_v, small = [], [], []
            for b in range(5):                                  # the host's rows as pages of its own
                r = torch.cat([rows[l][b], torch.zeros(2, -lens[b] % page, kv, dh, dtype=c.dtype)], 1)
                small.append(list(range(len(pool_k), len(pool_k) + r.shape[1] // page)) or [0])
                for j in range(r.shape[1] // page):
                    pool_k.append(r[0, j * page:(j + 1) * page].transpose(0, 1))
                    pool_v.append(r[1, j * page:(j + 1) * page].transpose(0, 1))
            if not pool_k:
                continue
            pk, pv = torch.stack(pool_k), torch.stack(pool_v)
            check_attention(c.attention(l, q.cuda()), q, pk, pv, small, lens, page, dtype)
            if turn % 3 == 2:
                bounds = torch.zeros(len(pk), kv, 2, dh, dtype=c.dtype)
                for b in range(5):
                    for j in range(-(-lens[b] // page)):
                        part = pk[small[b][j], :, :min(page, lens[b] - j * page)]
                        bounds[small[b][j], :, 0], bounds[small[b][j], :, 1] = part.amin(1), part.amax(1)
                picked = c.select(l, q.cuda(), 3)
                assert torch.equal(picked.cpu(), select_plain(q, bounds, small, lens, 3, page, kv))
                check_attention(c.attention(l, q.cuda(), blocks=picked), q, pk, pv, small, lens, page, dtype, blocks=picked.tolist())


def test_calls_in_a_captured_graph_and_on_another_stream():
    """Plan, store, choice and attention of a decoding turn captured once and replayed, eager turns in between; every replay
    against the eager calls on a copy."""
    page, kv, heads, dh = 16, 2, 8, 128
    def fresh():
        c, k, v, table, q = filled(BF16, heads, kv, dh, page, [600, 5, 0, 1300], spare=30, poison=False, extra_blocks=8)
        return c, q.cuda()
    a, q = fresh()
    e, _ = fresh()
    rows = torch.randn(4, 2, kv, dh, device="cuda").bfloat16()
    one = torch.ones(4, dtype=torch.int32, device="cuda")

    def turn(c, plan, stream=None):
        c.plan(one, out=plan, stream=stream)
        c.store(0, rows[:, 0], rows[:, 1], plan.slot, stream=stream)
        blocks = c.select(0, q, 6, stream=stream)
        return c.attention(0, q, stream=stream), c.attention(0, q, blocks=blocks, stream=stream), blocks

    pa, pe = a.new_plan(4, 4), e.new_plan(4, 4)
    turn(a, pa), turn(e, pe)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = turn(a, pa)
    side = torch.cuda.Stream()
    for i in range(8):
        rows.normal_()
        q.normal_()
        if i % 3 == 2:                                   # an eager turn of both, on a stream of its own
            side.wait_stream(torch.cuda.current_stream())
            x, y = turn(a, pa, side), turn(e, pe, side)
            torch.cuda.current_stream().wait_stream(side)
            assert all(torch.equal(p, r) for p, r in zip(x, y))
        graph.replay()
        want = turn(e, pe)
        for p, r in zip(got, want):
            assert torch.equal(p, r), i
        assert torch.equal(a.words, e.words) and torch.equal(a.k, e.k) and torch.equal(a.bounds, e.bounds)
    assert int(a.status) == 0


def test_calls_on_two_streams_at_once():
    """Workspaces and outputs come per call and stream: cut attention and long choices side by side give what they give alone."""
    caches = [filled(BF16, 8, 2, 64, 16, lens, seed=i, poison=False) for i, lens in enumerate(([20000, 300], [18000, 7]))]
    for c, *_ in caches:
        c.bounds.normal_()
    qs = [x[4].cuda() for x in caches]
    alone = [(c.attention(0, q), c.select(0, q, 100)) for (c, *_), q in zip(caches, qs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            got[i].append((caches[i][0].attention(0, qs[i], stream=s), caches[i][0].select(0, qs[i], 100, stream=s)))
    torch.cuda.synchronize()
    for i in range(2):
        for x, y in got[i]:
            assert torch.equal(x, alone[i][0]) and torch.equal(y, alone[i][1])


def test_graphs_and_eager_calls_do_not_share_a_workspace():
    """Two graphs captured one after the other, replayed at once on two streams next to eager calls on a third: cut attention of each
    keeps its own partial results."""
    caches = [filled(BF16, 8, 2, 64, 16, [20000 + 999 * i, 300], seed=i, poison=False) for i in range(3)]
    qs = [x[4].cuda() for x in caches]
    alone = [c.attention(0, q) for (c, *_), q in zip(caches, qs)]
    graphs, outs = [], []
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            outs.append(caches[i][0].attention(0, qs[i]))
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    eager = []
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
        eager.append(caches[2][0].attention(0, qs[2], stream=streams[2]))
    torch.cuda.synchronize()
    assert all(torch.equal(outs[i], alone[i]) for i in range(2)) and all(torch.equal(e, alone[2]) for e in eager)


def test_refusals_of_the_binding():
    c = B.PageCache(1, 8, 16, 2, 64, BF16, 3, 4)
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16, device="cuda")
    i32 = torch.zeros(3, dtype=torch.int32, device="cuda")
    bad = [lambda: c.plan(i32.long(), 3), lambda: c.plan(i32), lambda: c.plan(i32.cpu(), 3), lambda: c.plan(i32, out=c.new_plan(2, 3)),
           lambda: c.plan(torch.zeros(6, dtype=torch.int32, device="cuda")[::2], 3),
           lambda: c.store(0, q[:, :2].float(), q[:, :2], i32), lambda: c.store(0, q, q, i32), lambda: c.store(1, q[:, :2], q[:, :2], i32),
           lambda: c.store(0, q[:, :2], q[:, :2], i32[:2]), lambda: c.attention(0, q.float()), lambda: c.attention(0, q[:, :, :32]),
           lambda: c.attention(0, q[:, ::2]), lambda: c.attention(-1, q), lambda: c.attention(0, q, out=q[:2]),
           lambda: c.attention(0, q, blocks=i32.view(3, 1, 1)), lambda: c.select(0, q, 0), lambda: c.select(0, q, 5),
           lambda: c.select(0, q, 2, out=torch.zeros(3, 2, 3, dtype=torch.int32, device="cuda")), lambda: c.attention(0, q.cpu())]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            raise AssertionError(i)
    with pytest.raises(B.CerberusError):
        c.attention(0, torch.zeros(4, 4, 64, dtype=torch.bfloat16, device="cuda"))       # more sequences than the table
    with pytest.raises(B.CerberusError):
        c.attention(0, q[:, :3])                                                         # 3 heads on 2 key heads
    with pytest.raises(ValueError):
        B.PageCache(1, 8, 16, 2, 64, 7, 3, 4)
    with pytest.raises(ValueError):
        B.PageCache(1, 0, 16, 2, 64, BF16, 3, 4)
    with pytest.raises(ValueError):
        B.PageCache(1, 8, 16, 2, 64, BF16, 3, 4, device="cpu")


# ------------------------------------------------------------------------------------------------
# the step over pages
# ------------------------------------------------------------------------------------------------

def _pair(dtype, **kw):
    return H.Pair("tiny", dtype, "tiny", seed=0, max_batch=3, kv_capacity=192, **kw)


def _prompts(cfg, lens):
    return [synth.make_token_ids(n, cfg["vocab"], seed=10 + i) for i, n in enumerate(lens)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("page,bounds,heads", [(16, True, {}), (64, False, {}), (32, False, dict(n_heads=2, head_dim=128)),
                                              (16, True, dict(n_heads=2, head_dim=128))])
def test_paged_step_equals_the_step_over_the_slab(dtype, page, bounds, heads):
    """The same prompts go on in the slab (ar_step) and in pages: logits, tokens, lengths, gate and the cache rows they add.
    Same sums but for the attention's order: the tiny shape's tolerance of the step against the oracle."""
    pair = _pair(dtype, **heads)
    eng, cfg, lens, batch = pair.engine, pair.cfg, [37, 64, 5], 3
    tol = H.TOL_F32 if dtype == F32 else H.TOL_BF16_TINY
    st, sp = eng.new_state(), eng.new_state()
    for s in (st, sp):
        for b, p in enumerate(_prompts(cfg, lens)):
            eng.prefill(s, batch, b, p.to(torch.int32).cuda())
    cache = B.PageCache(cfg["n_layers"], 40, page, cfg["n_heads"], cfg["head_dim"], dtype, 4, 8, bounds=bounds)
    eng.move_prompts(sp, cache, lens)
    assert cache.kv_len.tolist() == lens + [0]
    sp.kv.fill_(float("nan"))                               # the step over pages does not touch the slab
    sp.kv_len.fill_(-1)
    taps = pair.taps()
    for i in range(5):
        sp.root_token.copy_(st.root_token)                  # (near-ties may part the two)
        eng.ar_step(st, batch)
        want = {k: getattr(taps, k).clone() for k in ("logits", "h_last", "node_token", "node_argmax", "head_logits")}
        eng.paged_step(sp, cache, batch)
        rows = torch.arange(batch, device="cuda") * pair.T
        assert (taps.logits[rows] - want["logits"][rows]).abs().max() <= tol.logits
        assert (taps.h_last[rows] - want["h_last"][rows]).abs().max() <= tol.hidden
        assert torch.equal(taps.node_token[rows], want["node_token"][rows])
        assert (taps.head_logits - want["head_logits"]).abs().max() <= tol.logits
        assert torch.equal(sp.accept_len, st.accept_len) and torch.equal(sp.accepted_tokens[:, 0], st.accepted_tokens[:, 0])
        assert (sp.entropy - st.entropy).abs().max() <= tol.entropy and torch.equal(sp.gate_flag, st.gate_flag)
        assert cache.kv_len.tolist()[:3] == st.kv_len.tolist() == [n + i + 1 for n in lens]
    for l in range(cfg["n_layers"]):
        for b, n in enumerate(lens):
            pos = torch.arange(n + 5, device="cuda")
            p = cache.block_table[b].long()[pos // page]
            for kvi, pool in ((0, cache.k), (1, cache.v)):
                got = pool[l][p, :, pos % page].transpose(0, 1).double().cpu().numpy()
                ref = st.kv[l, kvi, b, :, :n + 5].double().cpu().numpy()
                assert H.kv_mismatch(got, ref, tol) is None
    assert int(sp.status) == 0 and int(cache.status) == 0
    pair.engine.close()


@pytest.mark.parametrize("bounds", [True, False])
def test_paged_step_at_full_width(bounds):
    """The 7B shape's width and heads, two layers: the projection kernels that the small shape does not reach, 16 sequences of mixed
    lengths.  The bar of a step's logits against the oracle."""
    cfg = synth.make_config("7b", n_layers=2, vocab=1024, n_resblocks=1, special_block=-1)
    W = synth.make_weights(cfg, seed=1, dtype=torch.bfloat16, device="cuda")
    parent, rank = synth.make_tree("tiny", 4)
    eng = B.Engine(cfg, W, parent, rank, BF16, max_batch=16, kv_capacity=700)
    lens = [1 + 43 * b for b in range(16)]
    st = eng.new_state()
    for b, p in enumerate(_prompts(cfg, lens)):
        eng.prefill(st, 16, b, p.to(torch.int32).cuda())
    cache = B.PageCache(2, 600, 16, 32, 128, BF16, 16, 50, bounds=bounds)
    eng.move_prompts(st, cache, lens)
    taps = B.DeviceTaps(cfg, 16, len(parent))
    eng.set_taps(taps)
    rows = torch.arange(16, device="cuda") * len(parent)
    for _ in range(2):
        roots = st.root_token.clone()
        eng.paged_step(st, cache, 16)
        got, tokens = taps.logits[rows].clone(), st.accepted_tokens[:, 0].clone()
        st.root_token.copy_(roots)
        eng.ar_step(st, 16)
        assert (got - taps.logits[rows]).abs().max() <= H.TOL_BF16.logits and torch.equal(tokens, st.accepted_tokens[:, 0])
        assert torch.equal(cache.kv_len, st.kv_len)
    assert int(cache.status) == 0 and int(st.status) == 0
    eng.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_paged_step_sits_out_ends_and_runs_out_of_pages(dtype):
    pair = _pair(dtype)
    eng, cfg, lens = pair.engine, pair.cfg, [31, 16, 20]
    sp = eng.new_state()
    for b, p in enumerate(_prompts(cfg, lens)):
        eng.prefill(sp, 3, b, p.to(torch.int32).cuda())
    cache = B.PageCache(cfg["n_layers"], 5, 16, cfg["n_heads"], cfg["head_dim"], dtype, 3, 3, bounds=False)
    eng.move_prompts(sp, cache, lens)
    assert int(cache.n_free) == 0
    root = sp.root_token.clone()
    eng.paged_step(sp, cache, 3, torch.tensor([1, 1, 0], dtype=torch.int32, device="cuda"))
    assert sp.accept_len.tolist() == [1, 0, 0] and cache.kv_len.tolist() == [32, 16, 20]     # the second needs a page
    assert int(cache.status) == B.CERBERUS_DEV_KV_OVERFLOW and torch.equal(sp.root_token[1:], root[1:])
    cache.status.zero_()
    eng.paged_step(sp, cache, 3, torch.tensor([-1, 1, 1], dtype=torch.int32, device="cuda"))
    assert sp.accept_len.tolist() == [0, 1, 1] and cache.kv_len.tolist() == [0, 17, 21] and int(cache.status) == 0
    assert int(cache.n_free) == 1 and int(sp.accepted_tokens[1, 0]) == int(root[1])
    other = F32 if dtype == BF16 else BF16
    for bad in (B.PageCache(1, 5, 16, 4, 64, dtype, 3, 3), B.PageCache(cfg["n_layers"], 5, 16, 2, 64, dtype, 3, 3),
                B.PageCache(cfg["n_layers"], 5, 16, 4, 64, other, 3, 3)):
        with pytest.raises(ValueError):
            eng.paged_step(sp, bad, 3)
        with pytest.raises(ValueError):
            eng.move_prompts(sp, bad, [1, 1, 1])
    for lens_bad in ([1] * 4, [193], [-1], []):
        with pytest.raises(ValueError):
            eng.move_prompts(sp, cache, lens_bad)
    with pytest.raises(ValueError):
        eng.generate_paged(sp, cache, _prompts(cfg, [5, 5]), 1)                              # the second holds rows
    pages, table = cache.layers, cache.table                                                 # and from C
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    wrong = (B.Pages * 2)(*[B.Pages(p.k, p.v, p.bounds, p.n_pages, p.page_size, p.n_kv_heads, p.head_dim, 1 - dtype) for p in pages])
    with pytest.raises(B.CerberusError, match="layer 0"):
        B.cerberus_paged_step(eng.ctx, sp.struct, wrong, table, 3, None, 0, ws)
    with pytest.raises(B.CerberusError, match="batch"):
        B.cerberus_paged_step(eng.ctx, sp.struct, pages, table, 4, None, 0, ws)
    with pytest.raises(B.CerberusError, match="workspace"):
        B.cerberus_paged_step(eng.ctx, sp.struct, pages, table, 3, None, 0, ws[:256])
    with pytest.raises(B.CerberusError):
        eng.paged_step(sp, cache, 3, n_select=2)                                              # without bounds
    pair.engine.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_paged_step_over_chosen_blocks(dtype):
    """With room for every block the choice changes nothing but the order of sums; with fewer it stays finite and the rows
    kept are the same."""
    pair = _pair(dtype)
    eng, cfg, lens = pair.engine, pair.cfg, [150, 90, 33]
    tol = H.TOL_F32 if dtype == F32 else H.TOL_BF16_TINY
    taps, out = pair.taps(), {}
    for n_select in (0, 12, 4):
        sp = eng.new_state()
        for b, p in enumerate(_prompts(cfg, lens)):
            eng.prefill(sp, 3, b, p.to(torch.int32).cuda())
        cache = B.PageCache(cfg["n_layers"], 40, 16, cfg["n_heads"], cfg["head_dim"], dtype, 3, 12)
        eng.move_prompts(sp, cache, lens)
        eng.paged_step(sp, cache, 3, n_select=n_select)
        out[n_select] = taps.logits[torch.arange(3, device="cuda") * pair.T].clone()
        assert cache.kv_len.tolist() == [151, 91, 34] and sp.accept_len.tolist() == [1, 1, 1] and int(cache.status) == 0
    assert (out[12] - out[0]).abs().max() <= tol.logits
    assert torch.isfinite(out[4]).all() and (out[4][2] - out[0][2]).abs().max() <= tol.logits    # three blocks of four
    assert not torch.equal(out[4][0], out[0][0])
    pair.engine.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_paged_steps_leave_the_bounds_of_full_pages(dtype):
    """Twenty steps over page ends, blocks chosen: the bounds of every page that a sequence has left behind are its rows', whatever
    owned the page before, and a choice of the caller's on the same cache goes by them."""
    pair = _pair(dtype)
    eng, cfg, lens = pair.engine, pair.cfg, [40, 15, 1]
    sp = eng.new_state()
    for b, p in enumerate(_prompts(cfg, lens)):
        eng.prefill(sp, 3, b, p.to(torch.int32).cuda())
    cache = B.PageCache(cfg["n_layers"], 14, 16, cfg["n_heads"], cfg["head_dim"], dtype, 3, 8)
    cache.k.fill_(float("nan"))
    cache.v.fill_(float("nan"))
    cache.bounds.fill_(float("nan"))
    eng.move_prompts(sp, cache, lens)
    for i in range(20):
        eng.paged_step(sp, cache, 3, n_select=2 + i % 2)
    lens = [n + 20 for n in lens]
    assert cache.kv_len.tolist() == lens and int(cache.status) == 0
    for l in range(cfg["n_layers"]):
        for b, n in enumerate(lens):
            for p in cache.block_table[b, :n // 16].tolist():
                assert torch.equal(cache.bounds[l, p, :, 0], cache.k[l, p].amin(1)) and torch.equal(cache.bounds[l, p, :, 1], cache.k[l, p].amax(1))
        q = torch.randn(3, cfg["n_heads"], cfg["head_dim"], device="cuda").to(cache.dtype)
        for n_select in (1, 2, 3):
            assert torch.equal(cache.select(l, q, n_select).cpu(), select_plain(q.cpu(), cache.bounds[l].cpu(), cache.block_table.tolist(), lens, n_select, 16, cfg["n_heads"]))
    pair.engine.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_paged_step_in_a_captured_graph(dtype):
    """Steps captured once and replayed, eager steps in between, against eager steps on another cache."""
    pair = _pair(dtype)
    eng, cfg, lens = pair.engine, pair.cfg, [100, 7, 40]
    states = []
    for _ in range(2):
        sp = eng.new_state()
        for b, p in enumerate(_prompts(cfg, lens)):
            eng.prefill(sp, 3, b, p.to(torch.int32).cuda())
        cache = B.PageCache(cfg["n_layers"], 60, 16, cfg["n_heads"], cfg["head_dim"], dtype, 3, 10)
        eng.move_prompts(sp, cache, lens)
        eng.paged_step(sp, cache, 3, n_select=5)
        states.append((sp, cache))
    (a, ca), (e, ce) = states
    rows = torch.ones(3, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        eng.paged_step(a, ca, 3, rows, n_select=5)
    for i in range(8):
        rows.copy_(torch.tensor([1, i % 3 != 1, 1], dtype=torch.int32))
        if i % 3 == 2:
            eng.paged_step(a, ca, 3, rows)
            eng.paged_step(e, ce, 3, rows)
        graph.replay()
        eng.paged_step(e, ce, 3, rows, n_select=5)
        for n in ("root_token", "cand", "gate_flag", "entropy", "accept_len", "accepted_tokens", "status"):
            assert torch.equal(getattr(a, n), getattr(e, n)), (i, n)
        assert torch.equal(ca.words, ce.words) and torch.equal(ca.k, ce.k) and torch.equal(ca.v, ce.v) and torch.equal(ca.bounds, ce.bounds), i
    assert int(ca.status) == 0 and ca.kv_len.tolist() == [111, 15, 51]
    pair.engine.close()


def test_paged_step_without_a_page_number_of_the_pool():
    """A free list that names no page of the pool: the row is written nowhere and the status says so."""
    for bounds in (True, False):
        pair = _pair(BF16)
        eng, cfg = pair.engine, pair.cfg
        sp = eng.new_state()
        eng.prefill(sp, 1, 0, _prompts(cfg, [16])[0].to(torch.int32).cuda())
        cache = B.PageCache(cfg["n_layers"], 4, 16, cfg["n_heads"], cfg["head_dim"], BF16, 1, 3, bounds=bounds)
        eng.move_prompts(sp, cache, [16])
        kept = cache.k.clone(), cache.v.clone()
        cache.free_pages.fill_(5000)
        eng.paged_step(sp, cache, 1)
        assert int(cache.status) == B.CERBERUS_DEV_BAD_PAGE and torch.equal(cache.k, kept[0]) and torch.equal(cache.v, kept[1])
        pair.engine.close()


def test_generate_paged_equals_generate_without_the_tree():
    pair = _pair(F32, entropy_threshold=-1.0)               # the gate keeps every step on the one-token path
    eng, cfg = pair.engine, pair.cfg
    prompts = _prompts(cfg, [20, 60])
    want = eng.generate(eng.new_state(), prompts, 8)
    cache = B.PageCache(cfg["n_layers"], 16, 16, cfg["n_heads"], cfg["head_dim"], F32, 2, 8)
    for stream in (None, torch.cuda.Stream()):
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        got = eng.generate_paged(eng.new_state(), cache, prompts, 8, stream=stream)
        torch.cuda.synchronize()
        assert got == want and int(cache.n_free) == 16 and cache.kv_len.tolist() == [0, 0]
    pair.engine.close()


def test_entry_points_by_their_names():
    """The calls of the header, one by one, on tensors of the caller's own."""
    page, kv, heads, dh, n = 16, 2, 4, 64, 37
    i32 = dict(dtype=torch.int32, device="cuda")
    free, n_free, status = torch.arange(6, **i32), torch.tensor([6], **i32), torch.zeros(1, **i32)
    table, lens = torch.full((1, 4), -1, **i32), torch.zeros(1, **i32)
    pt = B.PageTable(table.data_ptr(), lens.data_ptr(), free.data_ptr(), n_free.data_ptr(), status.data_ptr(), 1, 4, page, 6)
    k, v = torch.zeros(6, kv, page, dh, device="cuda"), torch.zeros(6, kv, page, dh, device="cuda")
    bounds = torch.zeros(6, kv, 2, dh, device="cuda")
    pg = B.Pages(k.data_ptr(), v.data_ptr(), bounds.data_ptr(), 6, page, kv, dh, F32)
    row_start, first, slot = torch.zeros(2, **i32), torch.zeros(1, **i32), torch.zeros(n, **i32)
    B.cerberus_page_plan(pt, torch.tensor([n], **i32), n, row_start, first, slot)
    rows = torch.randn(n, 2, kv, dh, device="cuda")
    B.cerberus_page_store(pg, rows[:, 0], rows[:, 1], slot, status)
    q = torch.randn(1, heads, dh, device="cuda")
    ws = torch.empty(B.cerberus_paged_workspace_bytes(pg, pt, 1, heads, 2), dtype=torch.uint8, device="cuda")
    blocks, out = torch.zeros(1, kv, 2, **i32), torch.zeros(1, heads, dh, device="cuda")
    B.cerberus_page_select(pg, pt, q, blocks, ws)
    B.cerberus_paged_attention(pg, pt, q, out, 0.125, blocks, ws)
    assert table.tolist() == [[5, 4, 3, -1]] and int(status) == 0 and blocks.tolist() == [[[0, 2], [0, 2]]]
    check_attention(out, q.cpu(), k.cpu(), v.cpu(), table.tolist(), [n], page, F32, blocks=blocks.tolist())
