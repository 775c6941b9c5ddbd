"""The calls over pages by their own names refuse tensors whose type, shape or strides the library would take for others, on the CPU: a
stand-in for the library notes what gets through.  (Every tensor says that it lies on a GPU.)"""
import pytest
import torch

from paper_2410_13344_amd import binding as B


class OnGpu(torch.Tensor):
    """A tensor of the CPU that says it lies on a GPU."""
    is_cuda = True


def on(t):
    return t.as_subclass(OnGpu)


def ints(*shape):
    return on(torch.zeros(shape, dtype=torch.int32))


def rows(*shape, dtype=torch.bfloat16):
    return on(torch.zeros(shape, dtype=dtype))


class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*a):
            self.calls.append(name)
            return 0
        return call


@pytest.fixture
def library(monkeypatch):
    L = Library()
    monkeypatch.setattr(B, "_lib", L)
    return L


PAGES = B.Pages(4096, 4096, 4096, 8, 16, 2, 64, B.CERBERUS_BF16)
TABLE = B.PageTable(4096, 4096, 4096, 4096, 4096, 4, 8, 16, 8)
WS = on(torch.zeros(1024, dtype=torch.uint8))


def plan(new=ints(3), most=5, start=ints(4), first=ints(3), slot=ints(5)):
    B.cerberus_page_plan(TABLE, new, most, start, first, slot, stream=0)


def store(k=rows(5, 2, 64), v=rows(5, 2, 64), slot=ints(5), status=None):
    B.cerberus_page_store(PAGES, k, v, slot, status, stream=0)


def select(q=rows(3, 4, 64), blocks=ints(3, 2, 4), ws=WS):
    B.cerberus_page_select(PAGES, TABLE, q, blocks, ws, stream=0)


def attend(q=rows(3, 4, 64), out=rows(3, 4, 64), blocks=ints(3, 2, 4), ws=WS):
    B.cerberus_paged_attention(PAGES, TABLE, q, out, 0.125, blocks, ws, stream=0)


def step(new=ints(3), ws=WS):
    B.cerberus_paged_step(None, B.State(), PAGES, TABLE, 3, new, 0, ws, stream=0)


F32 = torch.float32
BAD = {
    "plan, int64 rows": lambda: plan(new=on(torch.zeros(3, dtype=torch.int64))),
    "plan, every other row": lambda: plan(new=ints(6)[::2]),
    "plan, row_start too short": lambda: plan(start=ints(3)),
    "plan, first_pos too short": lambda: plan(first=ints(2)),
    "plan, slots too few": lambda: plan(slot=ints(4)),
    "plan, strided slots": lambda: plan(slot=ints(10)[::2]),
    "store, other type of k": lambda: store(k=rows(5, 2, 64, dtype=F32)),
    "store, other type of v": lambda: store(v=rows(5, 2, 64, dtype=F32)),
    "store, columns apart": lambda: store(k=rows(5, 64, 2).transpose(1, 2)),
    "store, other heads": lambda: store(k=rows(5, 3, 64), v=rows(5, 3, 64)),
    "store, narrow rows": lambda: store(v=rows(5, 2, 32)),
    "store, fewer rows than slots": lambda: store(k=rows(4, 2, 64), v=rows(4, 2, 64)),
    "store, strided slots": lambda: store(slot=ints(10)[::2]),
    "store, float status": lambda: store(status=on(torch.zeros(1))),
    "select, int64 blocks": lambda: select(blocks=on(torch.zeros(3, 2, 4, dtype=torch.int64))),
    "select, blocks of other key heads": lambda: select(blocks=ints(3, 1, 4)),
    "select, blocks of fewer sequences": lambda: select(blocks=ints(2, 2, 4)),
    "select, strided blocks": lambda: select(blocks=ints(3, 2, 8)[:, :, ::2]),
    "select, other type of q": lambda: select(q=rows(3, 4, 64, dtype=F32)),
    "select, heads apart": lambda: select(q=rows(3, 8, 64)[:, ::2]),
    "select, strided workspace": lambda: select(ws=on(torch.zeros(2048, dtype=torch.uint8))[::2]),
    "attention, int64 blocks": lambda: attend(blocks=on(torch.zeros(3, 2, 4, dtype=torch.int64))),
    "attention, blocks of other key heads": lambda: attend(blocks=ints(3, 1, 4)),
    "attention, blocks of fewer sequences": lambda: attend(blocks=ints(2, 2, 4)),
    "attention, flat blocks": lambda: attend(blocks=ints(3, 8)),
    "attention, strided blocks": lambda: attend(blocks=ints(3, 4, 4)[:, ::2]),
    "attention, other type of q": lambda: attend(q=rows(3, 4, 64, dtype=F32)),
    "attention, other type of out": lambda: attend(out=rows(3, 4, 64, dtype=F32)),
    "attention, narrow rows": lambda: attend(q=rows(3, 4, 32), out=rows(3, 4, 32)),
    "attention, heads of out apart": lambda: attend(out=rows(3, 8, 64)[:, ::2]),
    "attention, columns apart": lambda: attend(q=rows(3, 64, 4).transpose(1, 2)),
    "attention, strided workspace": lambda: attend(ws=on(torch.zeros(2048, dtype=torch.uint8))[::2]),
    "step, rows of fewer sequences": lambda: step(new=ints(2)),
    "step, int64 rows": lambda: step(new=on(torch.zeros(3, dtype=torch.int64))),
    "step, strided rows": lambda: step(new=ints(6)[::2]),
}


@pytest.mark.parametrize("what", BAD)
def test_refused(library, what):
    with pytest.raises(AssertionError):
        BAD[what]()
    assert library.calls == []


GOOD = {
    "plan": plan, "store": store, "select": select, "attention": attend, "step": step,
    "plan, no room for slots": lambda: plan(most=0, slot=ints(1)),
    "plan, longer arrays": lambda: plan(start=ints(9), first=ints(9), slot=ints(9)),
    "store, rows and heads apart": lambda: store(k=rows(5, 2, 2, 64)[:, 0], v=rows(2, 5, 64).transpose(0, 1)),
    "store, status": lambda: store(status=ints(1)),
    "store, status of no dimension": lambda: store(status=ints(1)[0]),
    "select, a slice of a projection": lambda: select(q=rows(3, 12, 64)[:, 4:8]),
    "attention, all blocks": lambda: attend(blocks=None),
    "attention, rows apart": lambda: attend(q=rows(3, 12, 64)[:, 4:8], out=rows(3, 9, 64)[:, 1:5]),
    "attention, one query for all": lambda: attend(q=rows(1, 4, 64).expand(3, 4, 64)),
    "step, all": lambda: step(new=None),
    "step, rows of the largest batch": lambda: step(new=ints(4)),
}


@pytest.mark.parametrize("what", GOOD)
def test_accepted(library, what):
    GOOD[what]()
    assert len(library.calls) == 1
