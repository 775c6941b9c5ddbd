"""What the paged key-value cache's operators are measured on: a cache in pages that sequences share, what plans it, fills it
and reads it in the step of one token.

A case is a dict of plain values; `kind` names the operator:

  "plan"    cache.plan       which rows of which page the next rows of every sequence go to: block tables, lengths, free pages and
                             the slot of every new row.  `lens` rows held, `new` rows to come (-1: the sequence ends)
  "store"   cache.store      K/V rows into their slots, with the bounds (lowest, highest key coordinate) of the touched pages
  "attend"  cache.attention  attention of one new token per sequence over its pages, or over `select` blocks of each
                             (chosen beforehand) where that is above 0
  "select"  cache.select     the `select` best blocks of every sequence and key head by the bound of its queries on their keys

  heads, kv_heads, head_dim  head layout (kv_heads below heads: groups of queries share keys)
  page, pages, blocks        rows of a page, pages of the cache, blocks that a sequence's table has room for
  dtype                      "bf16" or "f32"

Lists of lengths are texts, "700,96,2048".  Head layouts, lengths and batches are those of the model shapes and benchmark of this
repository (32 or 4 heads of 128 or 64, up to 16 sequences of up to 4096 rows) and of serving in general (groups of four queries
to a key head, up to 256 requests, contexts of up to 131072 rows).  Everything is seeded: cache rows and queries N(0, 1), the keys
of a page around a mean of their own, pages handed out in random order.
"""
from __future__ import annotations

import random

import torch

own = False
_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_KV_OVERFLOW = 1            # bit of the status word: a sequence's rows found no place
_MOST_ROWS = 1 << 18        # cache rows of the largest attention, at eight key heads of 128 in bf16


def _ints(text):
    return [int(v) for v in str(text).split(",")]


def _text(values):
    return ",".join(str(v) for v in values)


def _spread(seed, n, lo, hi):
    """n lengths spread over the logarithm of a range, always the same ones."""
    rng = random.Random(seed)
    return [_log_int(rng, lo, hi) for _ in range(n)]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def _case(name, kind, **kw):
    c = dict(name=name, kind=kind, dtype="bf16", heads=32, kv_heads=32, head_dim=128, page=16, pages=0, blocks=0, lens="0", new="0", select=0)
    c.update(kw)
    lens, new = _ints(c["lens"]), _ints(c["new"])
    new = new * len(lens) if len(new) == 1 else new
    held = [-(-(v + max(n, 0)) // c["page"]) for v, n in zip(lens, new)]
    c["new"] = _text(new)
    c["blocks"] = c["blocks"] or max(1, max(held))
    c["pages"] = c["pages"] or max(1, sum(held))
    return c


def _plan_prompts():
    """256 places of a serving batch: most go on by a token, some end, some start a prompt."""
    rng = random.Random(5)
    lens, new = [], []
    for _ in range(256):
        what = rng.random()
        lens.append(0 if what < 0.15 else _log_int(rng, 16, 8192))
        new.append(_log_int(rng, 64, 8192) if what < 0.15 else -1 if what < 0.3 else 1)
    return _text(lens), _text(new)


def listed():
    prompts = _plan_prompts()
    return [
        # every step of plain decoding with the largest batch the decoder takes: a row each, now and then a page
        _case("plan_step_16", "plan", lens=_text(_spread(1, 16, 200, 4000)), new="1", pages=4096, blocks=256),
        # a busy server's turn: prompts start, sequences end, the others go on
        _case("plan_prompts_256", "plan", lens=prompts[0], new=prompts[1], pages=65536, blocks=1024),
        # what a decoding step stores in one layer of the 7B shape
        _case("store_step_16", "store", lens=_text(_spread(2, 16, 20, 120)), new="1"),
        # prompts moved into pages, one layer, eight key heads
        _case("store_prompts", "store", kv_heads=8, lens="0,0,0,37,0,0,250,0", new="1024,4096,333,2500,1,4096,1500,700", page=32),
        # the fp32 reference mode of the small shape: launches and latency
        _case("attend_tiny_f32", "attend", dtype="f32", heads=4, kv_heads=4, head_dim=64, lens="128"),
        # one sequence of the 7B shape, the headline prefix
        _case("attend_7b_l1024", "attend", lens="1025"),
        # the largest batch the decoder takes, ragged
        _case("attend_7b_batch16", "attend", lens="257,2049,512,1778,641,1302,1025,2000,334,1501,902,1889,2001,778,1101,1536"),
        # one long document, few key heads: only a split over its length fills the card
        _case("attend_long_131072", "attend", kv_heads=8, page=64, lens="131072"),
        # a server's batch, groups of four queries, lengths over two orders of magnitude, one place empty
        _case("attend_group4_batch64", "attend", kv_heads=8, lens=_text([0] + _spread(3, 63, 128, 16384))),
        # long documents, 32 blocks of 64 rows chosen of 512
        _case("attend_sparse_16x32768", "attend", kv_heads=8, page=64, lens=_text([32768 - 61 * i for i in range(16)]), select=32),
        # that choice
        _case("select_16x32768", "select", kv_heads=8, page=64, lens=_text([32768 - 61 * i for i in range(16)]), select=32),
        # a choice among few blocks, the batch of the serving benchmark
        _case("select_7b_batch8", "select", lens="1593,3313,1896,2684,2183,3057,1746,832", select=64),
    ]


def draw(rng: random.Random):
    """One more case of the same ranges; sizes over their logarithm, most of them odd."""
    kind = rng.choice(["plan", "store", "attend", "attend", "attend", "select"])
    page = rng.choice([16, 16, 32, 64, 128, 256])
    if kind == "plan":
        n = _log_int(rng, 1, 256)
        lens = [_log_int(rng, 1, 8192) - 1 for _ in range(n)]
        new = [rng.choice([1, 1, 1, 1, 0, -1, _log_int(rng, 2, 4096)]) for _ in range(n)]
        held = sum(-(-v // page) for v in lens)
        want = sum(max(w, 0) // page + 1 for w in new)
        c = _case("", kind, page=page, lens=_text(lens), new=_text(new), blocks=-(-12288 // page), pages=held + (want if rng.random() < 0.7 else want // 3))
        del c["name"]
        return c
    dtype, dh = rng.choice(["bf16", "bf16", "f32"]), rng.choice([128, 128, 64])
    kv, group = rng.choice([(32, 1), (40, 1), (4, 1), (8, 4), (8, 8), (2, 5), (1, 16), (4, 7), (1, 24)])
    heads = dict(dtype=dtype, head_dim=dh, heads=kv * group, kv_heads=kv, page=page)
    if kind == "store":
        n = _log_int(rng, 1, 64)
        most = max(2, 65536 // (kv * n))
        lens = [rng.choice([0, rng.randint(1, 3 * page)]) for _ in range(n)]
        c = _case("", kind, lens=_text(lens), new=_text([rng.choice([1, 1, _log_int(rng, 1, most), 0]) for _ in range(n)]), **heads)
        if max(_ints(c["new"])) < 1:
            c = _case("", kind, lens=_text(lens), new="1", **heads)
        del c["name"]
        return c
    n = _log_int(rng, 1, 40)
    most = max(2, min(131072, _MOST_ROWS * 8 // (n * kv * (2 if dtype == "f32" else 1))))
    lens = [_log_int(rng, 1, most) for _ in range(n)]
    if n > 2 and kind == "attend" and rng.random() < 0.4:
        lens[rng.randrange(n)] = 0
    blocks = -(-max(lens) // page)
    select = rng.randint(1, max(1, min(128, blocks))) if kind == "select" or rng.random() < 0.4 else 0
    c = _case("", kind, lens=_text(lens), select=select, **heads)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------
# what a program has in hand
# ------------------------------------------------------------------------------------------------

class _State:
    pass


def _tables(case, g):
    """Block tables of the sequences as they are now: pages in random order, the rest of them free."""
    lens, page, pages, blocks = _ints(case["lens"]), case["page"], case["pages"], case["blocks"]
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros((len(lens), blocks), dtype=torch.int32, device="cuda")
    held = torch.tensor([-(-v // page) for v in lens], device="cuda")
    first = torch.cumsum(held, 0) - held
    j = torch.arange(blocks, device="cuda")
    mine = j[None, :] < held[:, None]
    table[mine] = order[(first[:, None] + j[None, :])[mine]]
    used = int(held.sum())
    free = torch.zeros(pages, dtype=torch.int32, device="cuda")
    free[:pages - used] = order[used:]
    return table, torch.tensor(lens, dtype=torch.int32, device="cuda"), free, pages - used


def _pools(case, g):
    """K and V pages (one more than the case has: what the plain store of a row without a slot goes to)."""
    shape = (case["pages"] + 1, case["kv_heads"], case["page"], case["head_dim"])
    dt = _DTYPES[case["dtype"]]
    mean = torch.randn((shape[0], shape[1], 1, shape[3]), generator=g, device="cuda")
    k = torch.randn(shape, generator=g, device="cuda").mul_(0.8).add_(mean.mul_(0.6)).to(dt)
    v = torch.randn(shape, generator=g, device="cuda").to(dt)
    return k, v


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 17)
    s = _State()
    s.case, s.lens, s.new = case, _ints(case["lens"]), _ints(case["new"])
    n, kv, dh, page, dt = len(s.lens), case["kv_heads"], case["head_dim"], case["page"], _DTYPES[case["dtype"]]
    kind = case["kind"]
    table, lens, free, n_free = _tables(case, g)
    s.rows = sum(max(v, 0) for v in s.new)
    # the bookkeeping in one piece, so that a pass can put it back with one copy: free pages, status, lengths, free list, tables
    words = torch.cat([torch.tensor([n_free, 0], dtype=torch.int32, device="cuda"), lens, free, table.reshape(-1)])
    s.words, s.n_pages = words.clone(), case["pages"]
    s.new_rows = torch.tensor(s.new, dtype=torch.int32, device="cuda")
    cache = None
    if own:
        from paper_2410_13344_amd import binding as B

        code = B.CERBERUS_F32 if case["dtype"] == "f32" else B.CERBERUS_BF16
        cache = B.PageCache(0 if kind == "plan" else 1, case["pages"], page, kv, dh, code, n, case["blocks"])   # (a plan touches no layer)
        s.words = cache.words
        s.words.copy_(words)
    s.n_free, s.status = s.words[0:1], s.words[1:2]
    s.kv_len, s.free = s.words[2:2 + n], s.words[2 + n:2 + n + case["pages"]]
    s.table = s.words[2 + n + case["pages"]:].view(n, case["blocks"])
    s.cache = cache
    if kind == "plan":
        s.fresh = words
        if own:
            s.plan = cache.new_plan(n, max(1, s.rows))
        return s
    if kind == "select":
        # bounds of whole pages: what the stores of their rows left
        shape = (case["pages"], kv, 1, dh)
        mid = torch.randn(shape, generator=g, device="cuda").mul_(0.6)
        half = torch.rand(shape, generator=g, device="cuda").add_(0.8)
        s.bounds = torch.cat([mid - half, mid + half], dim=2).to(dt)
        s.q = torch.randn((n, case["heads"], dh), generator=g, device="cuda").to(dt)
        if own:
            cache.bounds[0].copy_(s.bounds)
        return s
    k, v = _pools(case, g)
    if own:
        cache.k[0].copy_(k[:-1])
        cache.v[0].copy_(v[:-1])
        k, v = cache.k[0], cache.v[0]
    s.k, s.v = k, v
    if kind == "store":
        s.bounds = torch.zeros((case["pages"] + 1, kv, 2, dh), dtype=dt, device="cuda")
        if own:
            cache.bounds.zero_()
            s.bounds = cache.bounds[0]
        # the tables as the plan of these rows left them, and its slots; the rows as a projection leaves them, K and V of a token together
        grown = dict(case, lens=_text([a + max(b, 0) for a, b in zip(s.lens, s.new)]))
        table, lens, free, n_free = _tables(grown, g)
        s.table.copy_(table)
        s.kv_len.copy_(lens)
        s.slot = torch.cat([table[b].long()[torch.arange(a, a + m, device="cuda") // page] * page + torch.arange(a, a + m, device="cuda") % page
                            for b, (a, m) in enumerate(zip(s.lens, s.new)) if m > 0]).to(torch.int32)
        rows = torch.randn((s.rows, 2, kv, dh), generator=g, device="cuda").to(dt)
        s.k_rows, s.v_rows = rows[:, 0], rows[:, 1]
        return s
    s.q = torch.randn((n, case["heads"], dh), generator=g, device="cuda").to(dt)
    s.blocks = None
    if case["select"]:
        picked = torch.full((n, kv, case["select"]), -1, dtype=torch.int32, device="cuda")
        for b, length in enumerate(s.lens):
            have = -(-length // page)
            take = min(have, case["select"])
            if take:
                score = torch.rand((kv, have), generator=g, device="cuda")
                score[:, have - 1] = 2.0
                picked[b, :, :take] = score.topk(take, dim=1).indices.sort(dim=1).values.to(torch.int32)
        s.blocks = picked
    return s


# ------------------------------------------------------------------------------------------------
# one pass: the framework's calls, or the plain forms
# ------------------------------------------------------------------------------------------------

def run(s):
    kind = s.case["kind"]
    if kind == "plan":
        s.words.copy_(s.fresh)                  # every pass starts from the same lengths and free pages
        if own:
            p = s.cache.plan(s.new_rows, out=s.plan)
            row_start, first_pos, slot = p.row_start, p.first_pos, p.slot
        else:
            row_start, first_pos, slot = _plan_plain(s)
        return {"n_free": s.n_free, "status": s.status, "kv_len": s.kv_len, "free": s.free, "table": s.table,
                "row_start": row_start, "first_pos": first_pos, "slot": slot}
    if kind == "store":
        if own:
            s.cache.store(0, s.k_rows, s.v_rows, s.slot)
            return {"k": s.k, "v": s.v, "bounds": s.bounds}
        _store_plain(s)
        return {"k": s.k[:-1], "v": s.v[:-1], "bounds": s.bounds[:-1]}
    if kind == "select":
        return s.cache.select(0, s.q, s.case["select"]) if own else _select_plain(s)
    return s.cache.attention(0, s.q, blocks=s.blocks) if own else _attend_plain(s)


def _plan_plain(s):
    page, pages, blocks, max_rows = s.case["page"], s.n_pages, s.case["blocks"], max(1, s.rows)
    dev = s.words.device
    L, new = s.kv_len.long(), s.new_rows.long()
    ends = new < 0
    held = (L + page - 1) // page
    j = torch.arange(blocks, device=dev)
    # pages of the sequences that end, pushed in order
    back = torch.where(ends, held, 0)
    at = torch.cumsum(back, 0) - back
    spot = torch.where(j[None, :] < back[:, None], s.n_free.long() + at[:, None] + j[None, :], pages)
    free = torch.cat([s.free, s.free.new_zeros(1)])
    free[spot.reshape(-1)] = s.table.reshape(-1)
    n_free = s.n_free.long() + back.sum()
    # rows and pages in order of the sequences
    rows = new.clamp(min=0)
    row_end = torch.cumsum(rows, 0)
    row_start = torch.cat([row_end.new_zeros(1), row_end])
    fits = ~ends & (L + new <= blocks * page) & (row_end <= max_rows)
    total = (L + rows + page - 1) // page
    need = torch.where(fits, total - held, 0)
    need_end = torch.cumsum(need, 0)
    granted = fits & ((need == 0) | (need_end <= n_free))
    need = torch.where(granted, need, 0)
    fresh = granted[:, None] & (j[None, :] >= held[:, None]) & (j[None, :] < total[:, None])
    source = n_free - 1 - ((need_end - need)[:, None] + j[None, :] - held[:, None])
    table = torch.where(fresh, free[source.clamp(0, pages - 1)], s.table)
    n_free = n_free - need.sum()
    first_pos = torch.where(granted, L, -1)
    # slots
    i = torch.arange(max_rows, device=dev)
    b = torch.searchsorted(row_end, i, right=True).clamp(max=len(s.lens) - 1)
    pos = L[b] + i - row_start[b]
    have = (i < row_end[-1]) & granted[b]
    slot = table[b, (pos // page).clamp(0, blocks - 1)].long() * page + pos % page
    slot = torch.where(have, slot, -1).to(torch.int32)
    refused = (~ends & ~granted).any()
    s.free.copy_(free[:pages])
    s.n_free.copy_(n_free)
    s.table.copy_(table)
    s.kv_len.copy_(torch.where(ends, 0, torch.where(granted, L + rows, L)))
    s.status.copy_(s.status | torch.where(refused, _KV_OVERFLOW, 0))
    return row_start.to(torch.int32), first_pos.to(torch.int32), slot


def _store_plain(s):
    page, pages = s.case["page"], s.n_pages
    slot = torch.where(s.slot < 0, pages * page, s.slot).long()
    p, off = slot // page, slot % page
    s.k[p, :, off] = s.k_rows
    s.v[p, :, off] = s.v_rows
    # rows that a touched page has now: those up to the furthest one stored
    filled = torch.zeros(pages + 1, dtype=torch.long, device=slot.device).scatter_reduce_(0, p, off + 1, "amax")
    for at in range(0, len(slot), 2048):
        pp = p[at:at + 2048]
        keys = s.k[pp].float()
        dead = (torch.arange(page, device=slot.device)[None, :] >= filled[pp][:, None])[:, None, :, None]
        s.bounds[pp, :, 0] = keys.masked_fill(dead, float("inf")).amin(2).to(s.bounds.dtype)
        s.bounds[pp, :, 1] = keys.masked_fill(dead, float("-inf")).amax(2).to(s.bounds.dtype)


def _select_plain(s):
    """Scores in 64 bits: two blocks next to the border change places with the last bits of a sum."""
    n, kv, dh, page, want = len(s.lens), s.case["kv_heads"], s.case["head_dim"], s.case["page"], s.case["select"]
    q = s.q.double().view(n, kv, -1, dh).sum(2)                     # the queries of a group, together
    out = torch.full((n, kv, want), -1, dtype=torch.int32, device=q.device)
    for b, length in enumerate(s.lens):
        have = -(-length // page)
        if have == 0:
            continue
        bounds = s.bounds[s.table[b, :have].long()].double()       # [blocks, kv, 2, dh]
        score = (torch.where(q[b] >= 0, bounds[:, :, 1], bounds[:, :, 0]) * q[b]).sum(-1).t().contiguous()
        score = torch.where(torch.isnan(score), float("inf"), score)
        rank = torch.zeros_like(score)
        rank[:, 0], rank[:, have - 1] = 1.0, 2.0                    # the first and the newest block come before all
        take = min(have, want)
        order = torch.sort(score, dim=1, descending=True, stable=True).indices
        order = torch.gather(order, 1, torch.sort(torch.gather(rank, 1, order), dim=1, descending=True, stable=True).indices)
        out[b, :, :take] = order[:, :take].sort(dim=1).values.to(torch.int32)
    return out


def _attend_plain(s):
    n, heads, kv, dh, page = len(s.lens), s.case["heads"], s.case["kv_heads"], s.case["head_dim"], s.case["page"]
    out = torch.zeros((n, heads, dh), dtype=s.q.dtype, device=s.q.device)
    scale = dh ** -0.5
    for b, length in enumerate(s.lens):
        if length == 0:
            continue
        have = -(-length // page)
        q = s.q[b].float().view(kv, -1, dh)
        if s.blocks is None:
            at = s.table[b, :have].long()
            k = s.k[at].permute(1, 0, 2, 3).reshape(kv, have * page, dh)[:, :length].float()
            v = s.v[at].permute(1, 0, 2, 3).reshape(kv, have * page, dh)[:, :length].float()
            x = torch.matmul(q, k.transpose(1, 2).contiguous()) * scale
        else:
            j = s.blocks[b].long()                                  # [kv, select]
            at = s.table[b][j.clamp(min=0)].long()
            h = torch.arange(kv, device=j.device)[:, None]
            pos = j[:, :, None] * page + torch.arange(page, device=j.device)
            dead = ((j < 0)[:, :, None] | (pos >= length)).reshape(kv, 1, -1)
            k = s.k[at, h].reshape(kv, -1, dh).float()
            v = s.v[at, h].reshape(kv, -1, dh).float()
            x = (torch.matmul(q, k.transpose(1, 2).contiguous()) * scale).masked_fill(dead, float("-inf"))
        w = torch.exp(x - x.amax(-1, keepdim=True))
        out[b] = (torch.matmul(w, v) / w.sum(-1, keepdim=True)).reshape(heads, dh).to(out.dtype)
    return out


# ------------------------------------------------------------------------------------------------
# from the definitions, in 64 bits
# ------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "plan":
        return _exact_plan(s)
    if case["kind"] == "store":
        return _exact_store(s)
    if case["kind"] == "select":
        return _exact_select(s)
    return _exact_attend(s)


def _exact_plan(s):
    """One sequence after the other, as the rule is worded."""
    page, blocks, max_rows = s.case["page"], s.case["blocks"], max(1, s.rows)
    free, table = s.free.tolist(), s.table.tolist()
    n_free, lens, status = int(s.n_free[0]), list(s.lens), 0
    for b, m in enumerate(s.new):
        if m < 0:
            for j in range(-(-lens[b] // page)):
                free[n_free] = table[b][j]
                n_free += 1
            lens[b] = 0
    row_start, first_pos, slot = [0], [], [-1] * max_rows
    asked, top = 0, n_free
    for b, m in enumerate(s.new):
        start = row_start[-1]
        row_start.append(start + max(m, 0))
        if m < 0:
            first_pos.append(-1)
            continue
        have, total = -(-lens[b] // page), -(-(lens[b] + m) // page)
        fits = lens[b] + m <= blocks * page and start + m <= max_rows
        if fits:
            asked += total - have
        if not fits or (total > have and asked > top):
            first_pos.append(-1)
            status |= _KV_OVERFLOW
            continue
        for j in range(have, total):
            n_free -= 1
            table[b][j] = free[n_free]
        first_pos.append(lens[b])
        for i in range(m):
            pos = lens[b] + i
            slot[start + i] = table[b][pos // page] * page + pos % page
        lens[b] += m
    out = {"n_free": [n_free], "status": [status], "kv_len": lens, "free": free, "table": table, "row_start": row_start,
           "first_pos": first_pos, "slot": slot}
    return {k: torch.tensor(v, dtype=torch.int32) for k, v in out.items()}


def _exact_store(s):
    page = s.case["page"]
    k, v, bounds = s.k[:s.n_pages].double(), s.v[:s.n_pages].double(), s.bounds[:s.n_pages].double()
    slots = s.slot.tolist()
    last = {}
    for slot in slots:
        if slot >= 0:
            last[slot // page] = max(last.get(slot // page, -1), slot % page)
    live = [i for i, slot in enumerate(slots) if slot >= 0]
    at = torch.tensor([slots[i] for i in live], device=k.device)
    rows = torch.tensor(live, device=k.device)
    kt, vt = k.permute(0, 2, 1, 3).reshape(-1, *k.shape[1::2]), v.permute(0, 2, 1, 3).reshape(-1, *v.shape[1::2])
    kt[at], vt[at] = s.k_rows.double()[rows], s.v_rows.double()[rows]
    k = kt.view(k.shape[0], page, *kt.shape[1:]).permute(0, 2, 1, 3)
    v = vt.view(v.shape[0], page, *vt.shape[1:]).permute(0, 2, 1, 3)
    for p, off in last.items():
        bounds[p] = torch.stack([k[p, :, :off + 1].min(dim=1).values, k[p, :, :off + 1].max(dim=1).values], dim=1)
    return {"k": k, "v": v, "bounds": bounds}


def _exact_select(s):
    case = s.case
    page, want, kv, group = case["page"], case["select"], case["kv_heads"], case["heads"] // case["kv_heads"]
    out = torch.full((len(s.lens), kv, want), -1, dtype=torch.int32)
    q = s.q.double()
    up, down = s.bounds[:, :, 1].double(), s.bounds[:, :, 0].double()
    for b, length in enumerate(s.lens):
        have = -(-length // page)
        if not have:
            continue
        pages = s.table[b, :have].long()
        for h in range(kv):
            total = torch.zeros(case["head_dim"], dtype=torch.float64, device=q.device)
            for g in range(group):
                total = total + q[b, h * group + g]
            score = (up[pages, h] @ total.clamp(min=0) + down[pages, h] @ total.clamp(max=0)).tolist()
            score[0] = float("inf")
            best = sorted(range(have - 1), key=lambda j: (-score[j], j))[:want - 1] + [have - 1]
            out[b, h, :len(best)] = torch.tensor(sorted(best), dtype=torch.int32)
    return out


def _exact_attend(s):
    case = s.case
    heads, kv, dh, page = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    out = torch.zeros((len(s.lens), heads, dh), dtype=torch.float64, device=s.q.device)
    for b, length in enumerate(s.lens):
        pos = torch.arange(length, device=s.q.device)
        page_of = s.table[b].long()[pos // page]
        for h in range(kv):
            rows, at = page_of, pos % page
            if s.blocks is not None:
                keep = torch.isin(pos // page, s.blocks[b, h].long())
                rows, at = rows[keep], at[keep]
            if not len(rows):
                continue
            k, v = s.k[rows, h, at].double(), s.v[rows, h, at].double()
            q = s.q[b].view(kv, -1, dh)[h].double()
            w = torch.softmax(q @ k.t().contiguous() / dh ** 0.5, dim=-1)
            out[b].view(kv, -1, dh)[h] = w @ v
    return out


# ------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------

def work(case):
    lens, new, page, kv, heads, dh = _ints(case["lens"]), _ints(case["new"]), case["page"], case["kv_heads"], case["heads"], case["head_dim"]
    elem = 4 if case["dtype"] == "f32" else 2
    n, kind = len(lens), case["kind"]
    if kind == "plan":
        rows = sum(max(m, 0) for m in new)
        moved = sum(-(-v // page) if m < 0 else -(-(v + m) // page) - -(-v // page) for v, m in zip(lens, new))
        return {"bytes": 4.0 * (5 * n + 2 * moved + rows), "flops": float(rows + moved)}
    if kind == "store":
        rows = sum(max(m, 0) for m in new)
        touched = sum(-(-(v + m) // page) - v // page for v, m in zip(lens, new) if m > 0)
        return {"bytes": float(4 * rows * kv * dh * elem + 2 * touched * kv * dh * elem + 4 * rows), "flops": 2.0 * rows * kv * dh}
    held = [-(-v // page) for v in lens]
    if kind == "select":
        blocks = sum(held)
        return {"bytes": float(blocks * kv * 2 * dh * elem + n * heads * dh * elem + 4 * blocks + 4 * n * kv * case["select"]),
                "flops": 2.0 * blocks * kv * dh}
    rows = [min(v, case["select"] * page) if case["select"] else v for v in lens]
    return {"bytes": float(sum(rows) * kv * dh * 2 * elem + 2 * n * heads * dh * elem + 4 * sum(-(-r // page) for r in rows)),
            "flops": float(4 * sum(rows) * heads * dh)}
