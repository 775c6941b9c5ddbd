"""One page cache, several host threads: calls that are more than one launch, or go through scratch memory, are not mixed up."""
import threading
import time

import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2410_13344_amd import binding as B
from paper_2410_13344_amd import synth
from tests import harness as H

BF16 = B.CERBERUS_BF16


class Recorder:
    """The library, but calls with scratch memory or tables take a while (and let go of the interpreter, as they do) and note
    who else is inside with the same memory."""

    def __init__(self, real):
        self.real, self.inside, self.mixed, self.calls, self.guard = real, {}, [], 0, threading.Lock()

    def __getattr__(self, name):
        return getattr(self.real, name)

    def _call(self, name, memory):
        with self.guard:
            self.calls += 1
            for m in memory:
                if self.inside.get(m, 0):
                    self.mixed.append(name)
                self.inside[m] = self.inside.get(m, 0) + 1
        time.sleep(0.02)
        with self.guard:
            for m in memory:
                self.inside[m] -= 1
        return 0

    def cerberus_page_plan(self, table, *a):
        return self._call("plan", ["table"])

    def cerberus_page_select(self, *a):
        return self._call("select", [("ws", a[8])])

    def cerberus_paged_attention(self, *a):
        return self._call("attention", [("ws", a[11])])

    def cerberus_paged_step(self, *a):
        return self._call("step", ["table", ("ws", a[7])])


def together(jobs):
    """Runs every job in a thread of its own, all beginning at once; what went wrong in them."""
    start, wrong = threading.Barrier(len(jobs)), []

    def go(job):
        try:
            start.wait()
            job()
        except Exception as e:                                   # (a thread's exception would only be printed)
            wrong.append(e)

    threads = [threading.Thread(target=go, args=(j,)) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    return wrong


def test_calls_of_threads_on_one_stream_do_not_overlap_in_memory(monkeypatch):
    pair = H.Pair("tiny", BF16, "tiny", seed=0, max_batch=1, kv_capacity=192)
    eng, cfg = pair.engine, pair.cfg
    cache = B.PageCache(cfg["n_layers"], 8, 16, cfg["n_heads"], cfg["head_dim"], BF16, 1, 4)
    st = eng.new_state()
    q = torch.zeros(1, cfg["n_heads"], cfg["head_dim"], dtype=torch.bfloat16, device="cuda")
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    cache.attention(0, q), cache.select(0, q, 2)                  # (sizes known, workspace there)
    torch.cuda.synchronize()
    rec = Recorder(B.lib())
    monkeypatch.setattr(B, "_lib", rec)
    jobs = []
    for i in range(2):
        jobs += [lambda: [cache.attention(0, q) for _ in range(4)], lambda: [cache.select(0, q, 2) for _ in range(4)],
                 lambda: [cache.plan(one, 1) for _ in range(4)], lambda: [eng.paged_step(st, cache, 1) for _ in range(4)],
                 lambda: [cache.attention(0, q, stream=side) for _ in range(4)]]
    wrong = together(jobs)
    monkeypatch.undo()
    assert not wrong and rec.calls == 40 and rec.mixed == [], (wrong, rec.mixed)
    eng.close()


def test_threads_that_call_at_once_get_what_they_get_alone():
    """Attention that is cut and joined and choices of two launches, from four threads on the stream that all of them have."""
    lens, page, kv, heads, dh = [20000, 300], 16, 2, 8, 64
    c = B.PageCache(1, 1300, page, kv, dh, BF16, 2, 1300)
    c.k.normal_(), c.v.normal_(), c.bounds.normal_()
    c.block_table.copy_(torch.randint(0, 1300, (2, 1300), device="cuda"))
    c.kv_len.copy_(torch.tensor(lens))
    qs = [torch.randn(2, heads, dh, device="cuda").bfloat16() for _ in range(4)]
    alone = [(c.attention(0, q), c.select(0, q, 100)) for q in qs]
    got = [[] for _ in qs]
    torch.cuda.synchronize()
    wrong = together([lambda i=i: [got[i].append((c.attention(0, qs[i]), c.select(0, qs[i], 100))) for _ in range(50)] for i in range(4)])
    torch.cuda.synchronize()
    assert not wrong
    for i in range(4):
        for out, blocks in got[i]:
            assert torch.equal(out, alone[i][0]) and torch.equal(blocks, alone[i][1]), i


def test_plans_of_threads_on_one_stream_hand_every_page_out_once():
    """Plans of many rows are two launches; four threads grow sequences of one cache at once."""
    c = B.PageCache(0, 4 * 40 * 3, 16, 1, 64, BF16, 1, 480)
    plans = [[c.new_plan(1, 2100) for _ in range(30)] for _ in range(4)]
    rows = torch.tensor([16], dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    wrong = together([lambda i=i: [c.plan(rows, out=p) for p in plans[i]] for i in range(4)])
    torch.cuda.synchronize()
    assert not wrong and int(c.status) == 0 and c.kv_len.tolist() == [4 * 30 * 16] and int(c.n_free) == 360
    slots = torch.cat([p.slot[:16] for ps in plans for p in ps]).tolist()
    assert len(set(slots)) == len(slots) == 4 * 30 * 16
