"""ctypes binding of libcerberus.so: the same entry points as include/cerberus.h, argument
marshalling only.  PyTorch supplies device memory and the stream; every step of the path runs in
the library's HIP kernels.  There is no fallback: a missing library is an error."""
from __future__ import annotations

import ctypes as C
import os
import threading
from typing import Optional, Sequence

import torch


_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcerberus.so")

CERBERUS_F32, CERBERUS_BF16 = 0, 1
CERBERUS_DEV_KV_OVERFLOW, CERBERUS_DEV_BAD_TOKEN, CERBERUS_DEV_LOG_FULL, CERBERUS_DEV_BAD_PAGE = 1, 2, 4, 8   # bits of the device status word
CERBERUS_MAX_TREE, CERBERUS_MAX_HEADS, CERBERUS_MAX_TOPK, CERBERUS_MAX_BATCH = 192, 8, 16, 16
CERBERUS_MAX_SEQS = 1024
DEV_KV_OVERFLOW, DEV_BAD_TOKEN = 1, 2

c_i32p = C.POINTER(C.c_int32)
c_f32p = C.POINTER(C.c_float)
c_vpp = C.POINTER(C.c_void_p)


class Config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "n_layers", "d_model", "n_heads", "head_dim", "d_ffn", "vocab", "n_cerb_heads", "n_resblocks",
        "special_block", "dtype", "max_batch", "kv_capacity", "topk")] + [
        ("rms_eps", C.c_float), ("rope_theta", C.c_float), ("entropy_threshold", C.c_float)]


class Weights(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("final_norm", C.c_void_p), ("lm_head", C.c_void_p),
                ("attn_norm", c_vpp), ("wqkv", c_vpp), ("wo", c_vpp), ("ffn_norm", c_vpp),
                ("w_gate_up", c_vpp), ("w_down", c_vpp), ("res_w", c_vpp), ("res_b", c_vpp),
                ("head_fc", c_vpp)]


class Tree(C.Structure):
    _fields_ = [("n_nodes", C.c_int32), ("parent", c_i32p), ("rank", c_i32p)]


class State(C.Structure):
    _fields_ = [("kv", C.c_void_p), ("kv_len", C.c_void_p), ("root_token", C.c_void_p), ("cand", C.c_void_p),
                ("gate_flag", C.c_void_p), ("entropy", C.c_void_p), ("accept_len", C.c_void_p),
                ("accepted_tokens", C.c_void_p), ("accepted_nodes", C.c_void_p), ("status", C.c_void_p)]


class Taps(C.Structure):
    _fields_ = [("logits", C.c_void_p), ("h_last", C.c_void_p), ("head_logits", C.c_void_p),
                ("node_token", C.c_void_p), ("node_argmax", C.c_void_p), ("forced_node_argmax", C.c_void_p),
                ("forced_gate_hidden", C.c_void_p)]


class Pages(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("bounds", C.c_void_p)] + [
        (n, C.c_int32) for n in ("n_pages", "page_size", "n_kv_heads", "head_dim", "dtype")]


class PageTable(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("block_table", "kv_len", "free_pages", "n_free", "status")] + [
        (n, C.c_int32) for n in ("max_seqs", "max_blocks", "page_size", "n_pages")]


_lib = None


def lib() -> C.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is not built: run `python -c 'import __graft_entry__ as g; g.build()'` "
                "(or python paper_2410_13344_amd/build.py) first; there is no CPU fallback")
        L = C.CDLL(LIB_PATH)
        L.cerberus_workspace_bytes.restype = C.c_size_t
        L.cerberus_workspace_bytes.argtypes = [C.POINTER(Config), C.POINTER(Tree)]
        L.cerberus_init.restype = C.c_int
        L.cerberus_init.argtypes = [C.POINTER(C.c_void_p), C.POINTER(Config), C.POINTER(Weights), C.POINTER(Tree),
                                    C.c_void_p, C.c_size_t]
        for name in ("cerberus_verify_step", "cerberus_ar_step"):
            f = getattr(L, name)
            f.restype = C.c_int
            f.argtypes = [C.c_void_p, C.POINTER(State), C.c_int32, C.c_void_p]
        L.cerberus_prefill.restype = C.c_int
        L.cerberus_prefill.argtypes = [C.c_void_p, C.POINTER(State), C.c_int32, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p]
        L.cerberus_decode.restype = C.c_int
        L.cerberus_decode.argtypes = [C.c_void_p, C.POINTER(State), C.c_int32, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p,
                                      C.c_void_p]
        L.cerberus_gate.restype = C.c_int
        L.cerberus_gate.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
        L.cerberus_accept.restype = C.c_int
        L.cerberus_accept.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(State), C.c_int32, C.c_void_p]
        L.cerberus_accept_noalloc.restype = C.c_int
        L.cerberus_accept_noalloc.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(State), C.c_int32, C.c_void_p]
        pages, table, i32, i64, vp = C.POINTER(Pages), C.POINTER(PageTable), C.c_int32, C.c_int64, C.c_void_p
        L.cerberus_page_plan.restype = C.c_int
        L.cerberus_page_plan.argtypes = [table, vp, i32, i32, vp, vp, vp, vp]
        L.cerberus_page_store.restype = C.c_int
        L.cerberus_page_store.argtypes = [pages, vp, i64, i64, vp, i64, i64, vp, i32, vp, vp]
        L.cerberus_paged_workspace_bytes.restype = C.c_size_t
        L.cerberus_paged_workspace_bytes.argtypes = [pages, table, i32, i32, i32]
        L.cerberus_page_select.restype = C.c_int
        L.cerberus_page_select.argtypes = [pages, table, vp, i64, i32, i32, i32, vp, vp, C.c_size_t, vp]
        L.cerberus_paged_attention.restype = C.c_int
        L.cerberus_paged_attention.argtypes = [pages, table, vp, i64, vp, i64, i32, i32, C.c_float, vp, i32, vp, C.c_size_t, vp]
        L.cerberus_paged_step.restype = C.c_int
        L.cerberus_paged_step.argtypes = [C.c_void_p, C.POINTER(State), pages, table, i32, vp, i32, vp, C.c_size_t, vp]
        L.cerberus_set_taps.restype = C.c_int
        L.cerberus_set_taps.argtypes = [C.c_void_p, C.POINTER(Taps)]
        L.cerberus_set_param.restype = C.c_int
        L.cerberus_set_param.argtypes = [C.c_void_p, C.c_char_p, C.c_int32]
        L.cerberus_bench_gemm.restype = C.c_int
        L.cerberus_bench_gemm.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.POINTER(C.c_double)]
        L.cerberus_last_error.restype = C.c_char_p
        L.cerberus_last_error.argtypes = []
        L.cerberus_destroy.restype = None
        L.cerberus_destroy.argtypes = [C.c_void_p]
        _lib = L
    return _lib


class CerberusError(RuntimeError):
    def __init__(self, code: int):
        self.code = code
        super().__init__(f"cerberus status {code}: {lib().cerberus_last_error().decode()}")


def _check(rc: int) -> None:
    if rc != 0:
        raise CerberusError(rc)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream_ptr(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream if type(stream) is int else stream.cuda_stream


def make_config(cfg: dict, dtype: int, max_batch: int, kv_capacity: int) -> Config:
    return Config(cfg["n_layers"], cfg["d_model"], cfg["n_heads"], cfg["head_dim"], cfg["d_ffn"], cfg["vocab"],
                  cfg["n_cerb_heads"], cfg["n_resblocks"], cfg["special_block"], dtype, max_batch, kv_capacity,
                  cfg["topk"], cfg["rms_eps"], cfg["rope_theta"], cfg["entropy_threshold"])


def make_tree(parent: Sequence[int], rank: Sequence[int]):
    n = len(parent)
    p = (C.c_int32 * n)(*parent)
    r = (C.c_int32 * n)(*rank)
    return Tree(n, C.cast(p, c_i32p), C.cast(r, c_i32p)), (p, r)


def _ptr_array(tensors):
    arr = (C.c_void_p * len(tensors))(*[t.data_ptr() for t in tensors])
    return C.cast(arr, c_vpp), arr


def make_weights(W: dict):
    """W: the dict of device tensors produced by synth.make_weights.  Returns (struct, keepalive).  The keepalive holds the
    matrices of the layers and the heads until cerberus_init is done with them; `embed` (fp32 mode: `lm_head` too), which a context
    reads at the caller's address on every step, is the caller's to keep alive, as the header says."""
    keep = []

    def arr(ts):
        p, a = _ptr_array(ts)
        keep.append(a)
        keep.append(ts)
        return p

    L = W["layers"]
    res_w = [b["w"] for h in W["heads"] for b in h["blocks"]]
    res_b = [b["b"] for h in W["heads"] for b in h["blocks"]]
    ws = Weights(W["embed"].data_ptr(), W["final_norm"].data_ptr(), W["lm_head"].data_ptr(),
                 arr([l["attn_norm"] for l in L]), arr([l["wqkv"] for l in L]), arr([l["wo"] for l in L]),
                 arr([l["ffn_norm"] for l in L]), arr([l["w_gate_up"] for l in L]), arr([l["w_down"] for l in L]),
                 arr(res_w), arr(res_b), arr([h["fc"] for h in W["heads"]]))
    return ws, keep


# ------------------------------------------------------------------------------------------------
# the entry points, named as in the header
# ------------------------------------------------------------------------------------------------

def cerberus_workspace_bytes(cfg: Config, tree: Tree) -> int:
    return int(lib().cerberus_workspace_bytes(C.byref(cfg), C.byref(tree)))


def cerberus_init(cfg: Config, weights: Weights, tree: Tree, workspace: torch.Tensor) -> int:
    ctx = C.c_void_p()
    _check(lib().cerberus_init(C.byref(ctx), C.byref(cfg), C.byref(weights), C.byref(tree), workspace.data_ptr(),
                               workspace.numel() * workspace.element_size()))
    return ctx.value


def cerberus_verify_step(ctx: int, state: State, batch: int, stream=None) -> None:
    _check(lib().cerberus_verify_step(ctx, C.byref(state), batch, _stream_ptr(stream)))


def cerberus_ar_step(ctx: int, state: State, batch: int, stream=None) -> None:
    _check(lib().cerberus_ar_step(ctx, C.byref(state), batch, _stream_ptr(stream)))


def cerberus_prefill(ctx: int, state: State, batch: int, seq: int, tokens: torch.Tensor, stream=None) -> None:
    assert tokens.dtype == torch.int32 and tokens.is_cuda and tokens.dim() == 1
    _check(lib().cerberus_prefill(ctx, C.byref(state), batch, seq, tokens.data_ptr(), tokens.shape[0], _stream_ptr(stream)))


def cerberus_decode(ctx: int, state: State, batch: int, n_steps: int, out_tokens: torch.Tensor, out_count: torch.Tensor,
                    stream=None) -> None:
    _check(lib().cerberus_decode(ctx, C.byref(state), batch, n_steps, out_tokens.data_ptr(), out_tokens.shape[1],
                                 out_count.data_ptr(), _stream_ptr(stream)))


def cerberus_gate(ctx: int, hidden: torch.Tensor, entropy_out: torch.Tensor, flag_out: torch.Tensor, stream=None) -> None:
    _check(lib().cerberus_gate(ctx, hidden.data_ptr(), hidden.shape[0], entropy_out.data_ptr(), flag_out.data_ptr(),
                               _stream_ptr(stream)))


def cerberus_accept(ctx: int, node_argmax: torch.Tensor, node_token: torch.Tensor, state: State, batch: int,
                    stream=None) -> None:
    _check(lib().cerberus_accept(ctx, node_argmax.data_ptr(), node_token.data_ptr(), C.byref(state), batch,
                                 _stream_ptr(stream)))


def cerberus_accept_noalloc(ctx: int, node_argmax: torch.Tensor, node_token: torch.Tensor, state: State, batch: int,
                            stream=None) -> None:
    _check(lib().cerberus_accept_noalloc(ctx, node_argmax.data_ptr(), node_token.data_ptr(), C.byref(state), batch,
                                         _stream_ptr(stream)))


# The calls over pages take sizes and strides from their tensors; what the kernels would read or write past a tensor's end, or take for
# another type, is refused here.

def _page_ints(t: torch.Tensor, *shape: int) -> bool:
    return t.is_cuda and t.dtype == torch.int32 and t.is_contiguous() and tuple(t.shape) == shape


def _page_rows(t: torch.Tensor, pages: Pages, heads: int, dense: bool) -> bool:
    """[rows][heads][head_dim] of the pages' type, a row's heads one after the other if `dense`."""
    return (t.is_cuda and t.dtype == (torch.float32 if pages.dtype == CERBERUS_F32 else torch.bfloat16) and t.dim() == 3 and
            t.shape[1] == heads and t.shape[2] == pages.head_dim and t.stride(2) == 1 and
            (not dense or heads == 1 or t.stride(1) == pages.head_dim))


def cerberus_page_plan(table: PageTable, new_rows: torch.Tensor, max_rows: int, row_start: torch.Tensor, first_pos: torch.Tensor,
                       slot: torch.Tensor, stream=None) -> None:
    assert all(t.is_cuda and t.dtype == torch.int32 and t.dim() == 1 and t.is_contiguous() for t in (new_rows, row_start, first_pos, slot))
    batch = new_rows.shape[0]
    assert row_start.shape[0] > batch and first_pos.shape[0] >= batch and slot.shape[0] >= max_rows
    _check(lib().cerberus_page_plan(table, new_rows.data_ptr(), batch, max_rows, row_start.data_ptr(), first_pos.data_ptr(),
                                    slot.data_ptr(), _stream_ptr(stream)))


def cerberus_page_store(pages: Pages, k: torch.Tensor, v: torch.Tensor, slot: torch.Tensor, status: Optional[torch.Tensor] = None,
                        stream=None) -> None:
    assert _page_ints(slot, slot.shape[0]) and k.shape[0] == v.shape[0] == slot.shape[0]
    assert _page_rows(k, pages, pages.n_kv_heads, False) and _page_rows(v, pages, pages.n_kv_heads, False)
    assert status is None or (status.is_cuda and status.dtype == torch.int32 and status.numel() >= 1)
    _check(lib().cerberus_page_store(pages, k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(), v.stride(0), v.stride(1),
                                     slot.data_ptr(), slot.shape[0], _ptr(status), _stream_ptr(stream)))


def cerberus_paged_workspace_bytes(pages: Pages, table: PageTable, batch: int, n_heads: int, n_select: int = 0) -> int:
    return int(lib().cerberus_paged_workspace_bytes(pages, table, batch, n_heads, n_select))


def cerberus_page_select(pages: Pages, table: PageTable, q: torch.Tensor, blocks: torch.Tensor, workspace: torch.Tensor,
                         stream=None) -> None:
    assert workspace.is_cuda and workspace.is_contiguous() and _page_rows(q, pages, q.shape[1], True)
    assert _page_ints(blocks, q.shape[0], pages.n_kv_heads, blocks.shape[-1])
    _check(lib().cerberus_page_select(pages, table, q.data_ptr(), q.stride(0), q.shape[0], q.shape[1], blocks.shape[2],
                                      blocks.data_ptr(), workspace.data_ptr(), workspace.numel(), _stream_ptr(stream)))


def cerberus_paged_attention(pages: Pages, table: PageTable, q: torch.Tensor, out: torch.Tensor, scale: float,
                             blocks: Optional[torch.Tensor], workspace: torch.Tensor, stream=None) -> None:
    assert workspace.is_cuda and workspace.is_contiguous()
    assert out.shape == q.shape and _page_rows(q, pages, q.shape[1], True) and _page_rows(out, pages, q.shape[1], True)
    assert blocks is None or _page_ints(blocks, q.shape[0], pages.n_kv_heads, blocks.shape[-1])
    _check(lib().cerberus_paged_attention(pages, table, q.data_ptr(), q.stride(0), out.data_ptr(), out.stride(0), q.shape[0], q.shape[1],
                                          scale, _ptr(blocks), 0 if blocks is None else blocks.shape[2], workspace.data_ptr(),
                                          workspace.numel(), _stream_ptr(stream)))


def cerberus_paged_step(ctx: int, state: State, layers, table: PageTable, batch: int, new_rows: Optional[torch.Tensor], n_select: int,
                        workspace: torch.Tensor, stream=None) -> None:
    assert workspace.is_cuda and workspace.is_contiguous()
    assert new_rows is None or (_page_ints(new_rows, new_rows.shape[0]) and new_rows.shape[0] >= batch)
    _check(lib().cerberus_paged_step(ctx, C.byref(state), layers, table, batch, _ptr(new_rows), n_select, workspace.data_ptr(),
                                     workspace.numel(), _stream_ptr(stream)))


def cerberus_set_taps(ctx: int, taps: Optional[Taps]) -> None:
    _check(lib().cerberus_set_taps(ctx, C.byref(taps) if taps is not None else None))


def cerberus_set_param(ctx: int, name: str, value: int) -> None:
    _check(lib().cerberus_set_param(ctx, name.encode(), value))


def cerberus_bench_gemm(ctx: int, kind: int, rows: int, stream=None) -> float:
    nbytes = C.c_double(0.0)
    _check(lib().cerberus_bench_gemm(ctx, kind, rows, _stream_ptr(stream), C.byref(nbytes)))
    return nbytes.value


def cerberus_destroy(ctx: int) -> None:
    lib().cerberus_destroy(ctx)


# ------------------------------------------------------------------------------------------------
# allocation helpers (device memory comes from torch)
# ------------------------------------------------------------------------------------------------

class DeviceState:
    """Owns the device arrays of a cerberus_state for `max_batch` sequences."""

    def __init__(self, cfg: dict, dtype: int, max_batch: int, kv_capacity: int, device="cuda"):
        tdt = torch.float32 if dtype == CERBERUS_F32 else torch.bfloat16
        Hc, K = cfg["n_cerb_heads"], cfg["topk"]
        i32 = dict(dtype=torch.int32, device=device)
        self.kv = torch.zeros((cfg["n_layers"], 2, max_batch, cfg["n_heads"], kv_capacity, cfg["head_dim"]),
                              dtype=tdt, device=device)
        self.kv_len = torch.zeros(max_batch, **i32)
        self.root_token = torch.zeros(max_batch, **i32)
        self.cand = torch.zeros((max_batch, Hc, K), **i32)
        self.gate_flag = torch.zeros(max_batch, **i32)
        self.entropy = torch.zeros(max_batch, dtype=torch.float32, device=device)
        self.accept_len = torch.zeros(max_batch, **i32)
        self.accepted_tokens = torch.zeros((max_batch, Hc + 1), **i32)
        self.accepted_nodes = torch.zeros((max_batch, Hc + 1), **i32)
        self.status = torch.zeros(1, **i32)
        self.struct = State(*[getattr(self, n).data_ptr() for n, _ in State._fields_])


class DeviceTaps:
    def __init__(self, cfg: dict, max_batch: int, T: int, device="cuda", logits=True, forced_argmax=False,
                 forced_gate=False):
        f32 = dict(dtype=torch.float32, device=device)
        i32 = dict(dtype=torch.int32, device=device)
        R = max_batch * T
        self.logits = torch.zeros((R, cfg["vocab"]), **f32) if logits else None
        self.h_last = torch.zeros((R, cfg["d_model"]), **f32)
        self.head_logits = torch.zeros((max_batch, cfg["n_cerb_heads"], cfg["vocab"]), **f32)
        self.node_token = torch.zeros(R, **i32)
        self.node_argmax = torch.zeros(R, **i32)
        self.forced_node_argmax = torch.zeros(R, **i32) if forced_argmax else None
        self.forced_gate_hidden = torch.zeros((max_batch, cfg["d_model"]), **f32) if forced_gate else None
        self.struct = Taps(*[_ptr(getattr(self, n)) for n, _ in Taps._fields_])


class PagePlan:
    """Where a batch's new rows go (see cerberus_page_plan)."""

    def __init__(self, batch: int, max_rows: int, device="cuda"):
        i32 = dict(dtype=torch.int32, device=device)
        self.batch, self.max_rows, self.device = batch, max_rows, torch.device(device)
        self.row_start = torch.zeros(batch + 1, **i32)
        self.first_pos = torch.zeros(batch, **i32)
        self.slot = torch.full((max(max_rows, 1),), -1, **i32)
        self.pointers = self.row_start.data_ptr(), self.first_pos.data_ptr(), self.slot.data_ptr()


class PageCache:
    """A key-value cache in pages that up to max_seqs sequences share: the device arrays of a cerberus_page_table and of the
    cerberus_pages of n_layers layers.  max_blocks: blocks of a sequence at most.  The
    bookkeeping (free pages, status, lengths, tables) is one tensor, `words`: a copy of it is a snapshot of who owns which page.
    A call on another stream than torch's current one of the cache's device: pass it as `stream`, and order the streams as for
    any tensor.  Outputs and workspaces come from torch's allocator, on the call's stream; a workspace serves the calls of one
    stream, and a captured graph has its own, so calls on several streams, and graphs, do not share them.  Several threads may
    call: the launches of a call are enqueued together, never between those of another call on the same cache."""

    def __init__(self, n_layers: int, n_pages: int, page_size: int, n_kv_heads: int, head_dim: int, dtype: int, max_seqs: int,
                 max_blocks: int, bounds: bool = True, device="cuda"):
        if dtype not in (CERBERUS_F32, CERBERUS_BF16):
            raise ValueError("dtype must be CERBERUS_F32 or CERBERUS_BF16")
        if min(n_pages, page_size, n_kv_heads, head_dim, max_seqs, max_blocks) < 1 or n_layers < 0:
            raise ValueError("non-positive size of a page cache")
        self.dtype = torch.float32 if dtype == CERBERUS_F32 else torch.bfloat16
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError("a page cache lives on a HIP device")
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU: the Cerberus library only runs on a HIP device")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        device, self._index = self.device, self.device.index
        self.n_layers, self.n_pages, self.page_size, self.n_kv_heads, self.head_dim = n_layers, n_pages, page_size, n_kv_heads, head_dim
        self.max_seqs, self.max_blocks, self._scale = max_seqs, max_blocks, head_dim ** -0.5
        shape = (n_layers, n_pages, n_kv_heads, page_size, head_dim)
        self.k = torch.zeros(shape, dtype=self.dtype, device=device)
        self.v = torch.zeros(shape, dtype=self.dtype, device=device)
        self.bounds = torch.zeros((n_layers, n_pages, n_kv_heads, 2, head_dim), dtype=self.dtype, device=device) if bounds else None
        self.words = torch.zeros(2 + max_seqs + n_pages + max_seqs * max_blocks, dtype=torch.int32, device=device)
        at = 2 + max_seqs
        self.n_free, self.status, self.kv_len = self.words[0:1], self.words[1:2], self.words[2:at]
        self.free_pages = self.words[at:at + n_pages]
        self.block_table = self.words[at + n_pages:].view(max_seqs, max_blocks)
        self.n_free.fill_(n_pages)
        self.free_pages.copy_(torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device=device))   # page 0 is taken first
        self.table = PageTable(*[getattr(self, n).data_ptr() for n in ("block_table", "kv_len", "free_pages", "n_free", "status")],
                               max_seqs, max_blocks, page_size, n_pages)
        self.layers = (Pages * max(n_layers, 1))()
        for i in range(n_layers):
            self.layers[i] = Pages(self.k[i].data_ptr(), self.v[i].data_ptr(), self.bounds[i].data_ptr() if bounds else None,
                                   n_pages, page_size, n_kv_heads, head_dim, dtype)
        self._bytes, self._kept = {}, {}
        # ctypes lets other threads run during a call; one that is two launches (a plan, a cut attention, a long choice), or hands its
        # workspace on to the next on its stream, must not have another one's launches between its own
        self._enqueue = threading.RLock()
        self._refs = [C.byref(self.layers[i]) for i in range(n_layers)]      # (what ctypes makes of a struct on every call)
        self._table, self._status = C.byref(self.table), self.status.data_ptr()

    def new_plan(self, batch: int, max_rows: int) -> PagePlan:
        return PagePlan(batch, max_rows, self.device)

    def workspace_bytes(self, batch: int, n_heads: int, n_select: int = 0) -> int:
        key = (batch, n_heads, n_select)
        n = self._bytes.get(key)
        if n is None:
            n = cerberus_paged_workspace_bytes(self.layers[0], self.table, batch, n_heads, n_select)
            if n == 0:
                raise CerberusError(-2)
            self._bytes[key] = n
        return n

    # A call takes about as long on the host as the smallest kernels run, so the methods below check in few steps, and only a
    # call on a stream of its own, or from another device, pays for torch's context of it.
    def _elsewhere(self, stream) -> bool:
        return stream is not None or torch._C._cuda_getDevice() != self._index

    def _on(self, stream):
        """Makes the cache's device and the call's stream torch's current ones."""
        if stream is not None and stream.device != self.device:
            raise ValueError(f"a stream of {stream.device} for a cache on {self.device}")
        return torch.cuda.stream(torch.cuda.current_stream(self.device) if stream is None else stream)

    def _stream(self) -> int:
        return torch._C._cuda_getCurrentRawStream(self._index)

    def _workspace(self, nbytes: int, stream: int) -> torch.Tensor:
        """Of a call on torch's current stream: one per stream, kept, for calls that follow each other there; a graph gets its own."""
        if torch._C._cuda_isCurrentStreamCapturing():
            return torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        ws = self._kept.get(stream)
        if ws is None or ws.numel() < nbytes:
            ws = self._kept[stream] = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        return ws

    def _refuse(self, what: str, t: torch.Tensor, expected) -> None:
        raise ValueError(f"{what}: {t.dtype} {tuple(t.shape)} strides {t.stride()} on {t.device}, expected {expected} on {self.device}")

    def _ints(self, what: str, t: torch.Tensor, shape) -> None:
        if t.dtype is not torch.int32 or t.shape != shape or t.device != self.device or not t.is_contiguous():
            self._refuse(what, t, f"contiguous int32 {tuple(shape)}")

    def _layer(self, layer: int):
        if not 0 <= layer < self.n_layers:
            raise ValueError(f"layer {layer} out of 0..{self.n_layers - 1}")
        return self._refs[layer]

    def plan(self, new_rows: torch.Tensor, max_rows: Optional[int] = None, out: Optional[PagePlan] = None, stream=None) -> PagePlan:
        """Places for the next rows of sequences 0..len(new_rows)-1.  max_rows: room of the slot map (with `out`: that plan's)."""
        if self._elsewhere(stream):
            with self._on(stream):
                return self.plan(new_rows, max_rows, out)
        batch = new_rows.numel()
        self._ints("new_rows", new_rows, (batch,))
        if out is None:
            if max_rows is None:
                raise ValueError("plan needs max_rows or out")
            out = PagePlan(batch, max_rows, self.device)
        elif out.batch != batch or out.device != self.device or (max_rows is not None and max_rows != out.max_rows):
            raise ValueError("out is a plan of another batch, device or max_rows")
        with self._enqueue:
            _check(lib().cerberus_page_plan(self._table, new_rows.data_ptr(), batch, out.max_rows, *out.pointers, self._stream()))
        return out

    def store(self, layer: int, k: torch.Tensor, v: torch.Tensor, slot: torch.Tensor, stream=None) -> None:
        """Rows k, v [rows][n_kv_heads][head_dim] (any strides of rows and heads) into their slots."""
        if self._elsewhere(stream):
            with self._on(stream):
                return self.store(layer, k, v, slot)
        n = slot.numel()
        self._ints("slot", slot, (n,))
        shape = (n, self.n_kv_heads, self.head_dim)
        pages, ks, vs = self._layer(layer), k.stride(), v.stride()
        for what, t, s in (("k", k, ks), ("v", v, vs)):
            if t.dtype is not self.dtype or t.shape != shape or t.device != self.device or s[2] != 1:
                self._refuse(what, t, f"{self.dtype} {shape}, contiguous rows")
        if n:
            _check(lib().cerberus_page_store(pages, k.data_ptr(), ks[0], ks[1], v.data_ptr(), vs[0], vs[1], slot.data_ptr(), n,
                                             self._status, self._stream()))

    def _query(self, what: str, q: torch.Tensor):
        """batch, heads, row stride"""
        if q.dtype is self.dtype and q.device == self.device and q.dim() == 3:
            (batch, heads, dim), s = q.shape, q.stride()
            if dim == self.head_dim and s[2] == 1 and (heads == 1 or s[1] == dim):
                return batch, heads, s[0]
        self._refuse(what, q, f"{self.dtype} [batch][heads][{self.head_dim}], the heads of a row contiguous")

    def select(self, layer: int, q: torch.Tensor, n_select: int, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """The n_select blocks of every sequence and key head that q [batch][n_heads][head_dim] attends to."""
        if self._elsewhere(stream):
            with self._on(stream):
                return self.select(layer, q, n_select, out)
        batch, heads, row = self._query("q", q)
        pages, shape = self._layer(layer), (batch, self.n_kv_heads, n_select)
        if not 1 <= n_select <= self.max_blocks:
            raise ValueError(f"n_select {n_select} out of 1..{self.max_blocks}")
        nbytes, s = self.workspace_bytes(batch, heads, n_select), self._stream()
        if out is None:
            out = self.words.new_empty(shape)
        else:
            self._ints("out", out, shape)
        with self._enqueue:
            ws = self._workspace(nbytes, s)
            _check(lib().cerberus_page_select(pages, self._table, q.data_ptr(), row, batch, heads, n_select, out.data_ptr(),
                                              ws.data_ptr(), nbytes, s))
        return out

    def attention(self, layer: int, q: torch.Tensor, scale: Optional[float] = None, blocks: Optional[torch.Tensor] = None,
                  out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """softmax(scale q K^T) V of one token q [batch][n_heads][head_dim] per sequence; scale: 1 / sqrt(head_dim)."""
        if self._elsewhere(stream):
            with self._on(stream):
                return self.attention(layer, q, scale, blocks, out)
        batch, heads, row = self._query("q", q)
        pages, n_select, picked = self._layer(layer), 0, None
        if blocks is not None:
            n_select, picked = blocks.shape[-1], blocks.data_ptr()
            self._ints("blocks", blocks, (batch, self.n_kv_heads, n_select))
            if n_select < 1:
                raise ValueError("blocks must name at least one block")
        nbytes, s = self.workspace_bytes(batch, heads, n_select), self._stream()
        if out is None:
            out_row = heads * self.head_dim
            out = torch.empty_like(q) if row == out_row else q.new_empty(q.shape)
        else:
            out_batch, out_heads, out_row = self._query("out", out)
            if out_batch != batch or out_heads != heads or (batch > 1 and abs(out_row) < heads * self.head_dim):
                raise ValueError("out has another shape than q, or rows that overlap")
        with self._enqueue:
            ws = self._workspace(nbytes, s)
            _check(lib().cerberus_paged_attention(pages, self._table, q.data_ptr(), row, out.data_ptr(), out_row, batch, heads,
                                                  self._scale if scale is None else scale, picked, n_select, ws.data_ptr(), nbytes, s))
        return out


class Engine:
    """A context plus the buffers that must outlive it, but for W["embed"] (fp32 mode: and W["lm_head"]): keep W for as long as
    the engine runs.  An engine whose dict is gone reads whatever the allocator puts there next."""

    def __init__(self, cfg: dict, W: dict, parent, rank, dtype: int, max_batch: int, kv_capacity: int):
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU: the Cerberus library only runs on a HIP device")
        self.cfg, self.dtype, self.max_batch, self.kv_capacity = cfg, dtype, max_batch, kv_capacity
        self.T = len(parent)
        self.c_cfg = make_config(cfg, dtype, max_batch, kv_capacity)
        self.c_tree, self._tree_keep = make_tree(parent, rank)
        self.c_weights, self._w_keep = make_weights(W)
        nbytes = cerberus_workspace_bytes(self.c_cfg, self.c_tree)
        if nbytes == 0:
            raise CerberusError(-2)
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        self.ctx = cerberus_init(self.c_cfg, self.c_weights, self.c_tree, self.workspace)

    def new_state(self) -> DeviceState:
        return DeviceState(self.cfg, self.dtype, self.max_batch, self.kv_capacity)

    def verify_step(self, st: DeviceState, batch: int, stream=None):
        cerberus_verify_step(self.ctx, st.struct, batch, stream)

    def ar_step(self, st: DeviceState, batch: int, stream=None):
        cerberus_ar_step(self.ctx, st.struct, batch, stream)

    def prefill(self, st: DeviceState, batch: int, seq: int, tokens: torch.Tensor, stream=None):
        cerberus_prefill(self.ctx, st.struct, batch, seq, tokens, stream)

    def decode(self, st: DeviceState, batch: int, n_steps: int, out_tokens: torch.Tensor, out_count: torch.Tensor,
               stream=None):
        cerberus_decode(self.ctx, st.struct, batch, n_steps, out_tokens, out_count, stream)

    def _fits(self, st: DeviceState, cache: PageCache) -> None:
        if cache.n_layers != self.cfg["n_layers"] or cache.device != st.kv.device or cache.dtype != st.kv.dtype or \
                cache.n_kv_heads != self.cfg["n_heads"] or cache.head_dim != self.cfg["head_dim"]:
            raise ValueError("a page cache of another model, dtype or device")

    def paged_step(self, st: DeviceState, cache: PageCache, batch: int, new_rows: Optional[torch.Tensor] = None, n_select: int = 0,
                   stream=None):
        """ar_step with the cache in pages: new_rows[b] 1 decodes a token, 0 sits out, below 0 ends the sequence."""
        self._fits(st, cache)
        if new_rows is not None:
            cache._ints("new_rows", new_rows, (batch,))
        nbytes = cache.workspace_bytes(batch, self.cfg["n_heads"], n_select)
        with cache._on(stream), cache._enqueue:
            ws = cache._workspace(nbytes, cache._stream())
            cerberus_paged_step(self.ctx, st.struct, cache.layers, cache.table, batch, new_rows, n_select, ws)

    def move_prompts(self, st: DeviceState, cache: PageCache, lens: Sequence[int], stream=None) -> PagePlan:
        """Rows 0..lens[b]-1 of the slab's sequences (0: none) become the next rows of the page cache's: what a prompt phase
        leaves goes on in pages, and the slab's places are free for other prompts."""
        self._fits(st, cache)
        if not 1 <= len(lens) <= min(cache.max_seqs, self.max_batch) or min(lens) < 0 or max(lens) > self.kv_capacity:
            raise ValueError("lens do not fit the slab or the page cache")
        with cache._on(stream):
            plan = cache.plan(torch.tensor(lens, dtype=torch.int32, device=cache.device), sum(lens))
            at = 0
            for b, n in enumerate(lens):
                for l in range(cache.n_layers if n else 0):
                    kv = st.kv[l, :, b, :, :n]                     # [2][heads][n][head_dim]
                    cache.store(l, kv[0].transpose(0, 1), kv[1].transpose(0, 1), plan.slot[at:at + n])
                at += n
        return plan

    def generate_paged(self, st: DeviceState, cache: PageCache, prompts, n_steps: int, n_select: int = 0, stream=None):
        """Prompt phase in the slab, then n_steps one-token steps in pages; returns the committed token ids of every sequence
        (fewer where the pages ran out) and ends the sequences, the first of the cache: they must be empty."""
        batch = len(prompts)
        self._fits(st, cache)
        if not 1 <= batch <= min(cache.max_seqs, self.max_batch) or max(len(p) for p in prompts) > self.kv_capacity:
            raise ValueError("prompts do not fit the slab or the page cache")
        with cache._on(stream):
            if cache.kv_len[:batch].any():
                raise ValueError("the page cache's sequences are not empty")
            st.kv_len[:batch] = 0
            for b, p in enumerate(prompts):
                self.prefill(st, batch, b, p.to(device="cuda", dtype=torch.int32))
            self.move_prompts(st, cache, [len(p) for p in prompts])
            log = torch.full((batch, n_steps), -1, dtype=torch.int32, device="cuda")
            here = (cache.kv_len[:batch] > 0).to(torch.int32)      # a prompt that found no pages decodes nothing
            for i in range(n_steps):
                self.paged_step(st, cache, batch, here, n_select)
                log[:, i] = torch.where(st.accept_len[:batch] > 0, st.accepted_tokens[:batch, 0], -1)
            cache.plan(torch.full((batch,), -1, dtype=torch.int32, device="cuda"), 0)
            out = log.cpu()
        return [[t for t in row if t >= 0] for row in out.tolist()]

    def generate(self, st: DeviceState, prompts, n_steps: int, stream=None):
        """Prompt phase for every sequence, then n_steps chained decoding steps (Algorithm 1 from its
        first line to its last); returns the committed token ids of every sequence.  Only calls and
        buffers: everything is computed by cerberus_prefill and cerberus_decode."""
        batch = len(prompts)
        st.kv_len[:batch] = 0
        for b, p in enumerate(prompts):
            self.prefill(st, batch, b, p.to(device="cuda", dtype=torch.int32), stream)
        cap = n_steps * (self.cfg["n_cerb_heads"] + 1)
        log = torch.full((batch, cap), -1, dtype=torch.int32, device="cuda")
        count = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.decode(st, batch, n_steps, log, count, stream)
        torch.cuda.synchronize()
        return [log[b, :int(count[b])].cpu().tolist() for b in range(batch)]

    def set_taps(self, taps: Optional[DeviceTaps]):
        self._taps = taps
        cerberus_set_taps(self.ctx, taps.struct if taps is not None else None)

    def set_param(self, name: str, value: int):
        cerberus_set_param(self.ctx, name, value)

    def close(self):
        if self.ctx:
            cerberus_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
