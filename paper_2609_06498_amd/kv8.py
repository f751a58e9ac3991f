"""Paged KV cache in 8 bits: page tables sized to the requests (PagePool), the
append of key and value rows and the attention over them (KV8Cache).

Argument marshalling over dflow_page_resize, dflow_kv8_append and
dflow_kv8_attention; the layouts are theirs (include/dflow.h).  The tensors
belong to the caller and every call is asynchronous on torch's current stream
of their device.  Calls through one KV8Cache share its workspace, so they must
execute in order: one stream, or streams ordered by events; graphs captured
through one cache are replayed one at a time, and the cache outlives them.  What only the device can see
(a page id outside the pool, a sequence that does not fit) sets bits of the
object's status word, which status() reads.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

from .runtime import DFLOW_BF16, DFLOW_F32, KV8, PAGE, DFlowError, Pool, load_library

GROUP = 16                     # tokens per scale
WORKSPACE_ZEROED = 4096        # DFLOW_KV8_WORKSPACE_ZEROED


def _refuse(index, need):
    """Raises for the first of need = [(name, tensor, dtype, least shape or None)] that does not fit."""
    for name, t, dt, shape in need:
        if t.get_device() != index:
            raise DFlowError(f"{name} is on {t.device}, not on cuda:{index}")
        if dt is not None and (t.dtype is not dt or not t.is_contiguous()):
            raise DFlowError(f"{name} must be contiguous {dt}, got {t.dtype} with strides {t.stride()}")
        if shape is not None and (t.dim() != len(shape) or any(h < w for h, w in zip(t.shape, shape))):
            raise DFlowError(f"{name} has shape {tuple(t.shape)}, at least {shape} needed")


class _DeviceCalls:
    """Library calls on a device's current stream, with a status word."""

    def _open(self, t):
        import torch
        if t.device.type != "cuda":
            raise DFlowError("the 8-bit cache needs a HIP device; there is no CPU path")
        self.torch, self.device, self.index, self.lib = torch, t.device, t.get_device(), load_library()
        self.status_word = torch.zeros(1, dtype=torch.int32, device=t.device)
        self._status = self.status_word.data_ptr()
        # (a call takes a few microseconds on the device: its host side avoids what is slow in Python)
        self._raw_stream = torch._C._cuda_getCurrentRawStream
        self._current = torch._C._cuda_getDevice

    def _call(self, fn, *args):
        """fn(stream, *args) on the current stream of the tensors' device, made current if it is not."""
        if self._current() == self.index:
            rc = fn(self._raw_stream(self.index), *args)
        else:
            with self.torch.cuda.device(self.index):
                rc = fn(self._raw_stream(self.index), *args)
        if rc != 0:
            raise DFlowError(f"{fn.__name__} failed ({rc}): {self.lib.dflow_last_error().decode()}")

    def status(self, clear: bool = True) -> int:
        """DFLOW_STATUS_* bits set by the calls so far (waits for the current stream)."""
        with self.torch.cuda.device(self.index):
            v = int(self.status_word.item())
            if clear and v:
                self.status_word.zero_()
        return v


class PagePool(_DeviceCalls):
    """Page-table rows of a batch and the stack of free pages, on the device.

    page_table int32 [rows, max_pages], n_held int32 [rows], free_pages int32
    [num_pages] with its top at n_free[0] - 1, n_free int32 [1]."""

    def __init__(self, page_table, n_held, free_pages, n_free):
        self._open(page_table)
        i32 = self._i32 = self.torch.int32
        _refuse(self.index, [("page_table", page_table, i32, (1, 1)), ("free_pages", free_pages, i32, (1,)),
                             ("n_held", n_held, i32, (page_table.shape[0],)), ("n_free", n_free, i32, (1,))])
        self.page_table, self.n_held, self.free_pages, self.n_free = page_table, n_held, free_pages, n_free
        self.num_pages = free_pages.shape[0]
        self._pool = Pool(page_table.data_ptr(), page_table.shape[1], n_held.data_ptr(), free_pages.data_ptr(),
                          self.num_pages, n_free.data_ptr())
        self._ref = ctypes.byref(self._pool)

    @classmethod
    def alloc(cls, rows: int, max_pages: int, num_pages: int, device="cuda:0") -> "PagePool":
        """Empty rows and a stack of all pages, page 0 on top."""
        import torch
        i32 = lambda x: x.to(dtype=torch.int32, device=device)
        return cls(i32(torch.full((rows, max_pages), -1)), i32(torch.zeros(rows)),
                   i32(torch.arange(num_pages - 1, -1, -1)), i32(torch.tensor([num_pages])))

    def resize(self, seq_len, new_len=None, slot=None, row_start=None):
        """dflow_page_resize over the first len(seq_len) rows; with `slot` (int32
        [capacity]) also the slot map of the new tokens and their row_start
        [nseq + 1]."""
        n, i, i32 = len(seq_len), self.index, self._i32
        if n > self.page_table.shape[0]:
            raise DFlowError(f"{n} sequences, {self.page_table.shape[0]} page-table rows")
        given = seq_len if new_len is None else (seq_len, new_len) if slot is None else (seq_len, new_len, slot, row_start)
        if slot is not None and (new_len is None or row_start is None):
            raise DFlowError("a slot map needs new_len and row_start")
        if slot is None and row_start is not None:
            raise DFlowError("row_start comes with a slot map")
        cap = 0 if slot is None else slot.numel()
        for t in (given if type(given) is tuple else (given,)):
            if t.dtype is not i32 or t.get_device() != i or t.dim() != 1 or not t.is_contiguous():
                _refuse(i, [("seq_len", seq_len, i32, (1,))] + [(m, x, i32, (k,)) for m, x, k in (
                    ("new_len", new_len, n), ("slot", slot, 0), ("row_start", row_start, n + 1)) if x is not None])
        if new_len is not None and len(new_len) < n or slot is not None and len(row_start) < n + 1:
            raise DFlowError(f"new_len needs {n} and row_start {n + 1} entries")
        self._call(self.lib.dflow_page_resize, self._ref, n, seq_len.data_ptr(),
                   None if new_len is None else new_len.data_ptr(), None if slot is None else slot.data_ptr(), cap,
                   None if slot is None else row_start.data_ptr(), self._status)


class KV8Cache(_DeviceCalls):
    """One layer's 8-bit cache: k uint8 [num_pages, n_kv_heads, 64, head_dim],
    v uint8 [num_pages, n_kv_heads, head_dim, 64] (e4m3 codes), k_scale and
    v_scale fp32 [num_pages, n_kv_heads, 4]."""

    def __init__(self, k, v, k_scale, v_scale):
        self._open(k)
        torch = self.torch
        _refuse(self.index, [("v", v, None, None), ("k_scale", k_scale, None, None), ("v_scale", v_scale, None, None)])
        if k.dim() != 4 or k.shape[2] != PAGE:
            raise DFlowError(f"k has shape {tuple(k.shape)}, [num_pages, n_kv_heads, {PAGE}, head_dim] needed")
        n, h, _, d = k.shape
        for name, t, dt, shape in (("k", k, torch.uint8, (n, h, PAGE, d)), ("v", v, torch.uint8, (n, h, d, PAGE)),
                                   ("k_scale", k_scale, torch.float32, (n, h, PAGE // GROUP)),
                                   ("v_scale", v_scale, torch.float32, (n, h, PAGE // GROUP))):
            if t.dtype is not dt or tuple(t.shape) != shape or not t.is_contiguous():
                raise DFlowError(f"{name} must be contiguous {dt} of shape {shape}, got {t.dtype} {tuple(t.shape)}")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.num_pages, self.n_kv_heads, self.head_dim = n, h, d
        self._kv = KV8(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), n, h, d)
        self._ref = ctypes.byref(self._kv)
        self._scale = 1.0 / math.sqrt(d)
        self._codes = {torch.bfloat16: DFLOW_BF16, torch.float32: DFLOW_F32}
        self._i32 = torch.int32
        self._ws, self._ws_ptr, self._ws_bytes, self._kept = None, None, 0, []
        self._need = {}

    @classmethod
    def alloc(cls, num_pages: int, n_kv_heads: int, head_dim: int, device="cuda:0") -> "KV8Cache":
        """A cache of zeros with unit scales."""
        import torch
        u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8, device=device)
        one = lambda: torch.ones(num_pages, n_kv_heads, PAGE // GROUP, dtype=torch.float32, device=device)
        return cls(u8(num_pages, n_kv_heads, PAGE, head_dim), u8(num_pages, n_kv_heads, head_dim, PAGE), one(), one())

    def _rows(self, name, t, heads):
        """(rows, heads, dtype code, row stride in elements) of a [rows, heads, head_dim] tensor whose rows are dense."""
        code = self._codes.get(t.dtype)
        n, h, d = t.shape if t.dim() == 3 else (0, 0, 0)
        if code is None or d != self.head_dim or h < 1 or (heads is not None and h != heads):
            raise DFlowError(f"{name} must be bfloat16 or float32 [rows, {heads or 'heads'}, {self.head_dim}], got "
                             f"{t.dtype} {tuple(t.shape)}")
        if t.get_device() != self.index:
            _refuse(self.index, [(name, t, None, None)])
        if t.is_contiguous():
            return n, h, code, h * d
        s = t.stride()
        if s[2] != 1 or (h > 1 and s[1] != d):
            raise DFlowError(f"{name}: the heads of a row must be contiguous (strides {s})")
        return n, h, code, (s[0] if n > 1 else h * d)

    def append(self, k, v, slot):
        """dflow_kv8_append: rows k, v [rows, n_kv_heads, head_dim] (bf16 or fp32) to their slots (int32 [rows], -1: none)."""
        n, _, code, ld_k = self._rows("k", k, self.n_kv_heads)
        n_v, _, code_v, ld_v = self._rows("v", v, self.n_kv_heads)
        if code_v != code or n_v != n:
            raise DFlowError(f"k {k.dtype} {tuple(k.shape)} and v {v.dtype} {tuple(v.shape)} differ")
        if slot.dtype is not self._i32 or slot.get_device() != self.index or slot.numel() < n or not slot.is_contiguous():
            _refuse(self.index, [("slot", slot, self._i32, (n,))])
        self._call(self.lib.dflow_kv8_append, code, self._ref, n, k.data_ptr(), ld_k, v.data_ptr(), ld_v, slot.data_ptr(),
                   self._status)

    def _workspace(self, key):
        """Workspace for calls of these sizes.  A buffer that is outgrown is kept: graphs captured with it hold its address."""
        need = self.lib.dflow_kv8_attention_workspace(*key, self.n_kv_heads, self.head_dim)
        if need == ctypes.c_size_t(-1).value:
            raise DFlowError(f"dflow_kv8_attention_workspace: {self.lib.dflow_last_error().decode()}")
        if need > self._ws_bytes:
            if self.torch.cuda.is_current_stream_capturing():
                # (its first bytes would be zeroed by the graph's replays only)
                raise DFlowError("this call's workspace must exist before it is captured: run it once first")
            if self._ws is not None:
                self._kept.append(self._ws)
            self._ws_bytes = max(need, 2 * self._ws_bytes)
            self._ws = self.torch.empty(self._ws_bytes, dtype=self.torch.uint8, device=self.device)
            self._ws[:WORKSPACE_ZEROED].zero_()
            self._ws_ptr = self._ws.data_ptr()
        if len(self._need) >= 4096:
            self._need.clear()
        self._need[key] = need

    def attention(self, q, page_table, kv_len, row_start, max_rows: int, max_len: int, causal: bool = True,
                  scale: Optional[float] = None, out=None):
        """dflow_kv8_attention: q [rows, n_heads, head_dim] (bf16 or fp32) of
        len(kv_len) sequences, rows row_start[s] .. row_start[s + 1] - 1 each, over
        kv_len[s] cached tokens.  max_rows and max_len bound both.  scale
        defaults to head_dim^-1/2.  Returns out."""
        rows, heads, code, ld_q = self._rows("q", q, None)
        if out is None:
            out = self.torch.zeros(q.shape, dtype=q.dtype, device=q.device)
        rows_o, _, code_o, ld_o = self._rows("out", out, heads)
        if code_o != code or rows_o != rows:
            raise DFlowError(f"q {q.dtype} {tuple(q.shape)} and out {out.dtype} {tuple(out.shape)} differ")
        i, i32, n = self.index, self._i32, len(kv_len)
        width = page_table.shape[-1]
        if not (page_table.dtype is i32 and kv_len.dtype is i32 and row_start.dtype is i32
                and page_table.is_contiguous() and kv_len.is_contiguous() and row_start.is_contiguous()
                and page_table.get_device() == i and kv_len.get_device() == i and row_start.get_device() == i
                and page_table.dim() == 2 and len(page_table) >= n and len(row_start) > n):
            _refuse(i, [("page_table", page_table, i32, (n, 1)), ("kv_len", kv_len, i32, (1,)),
                        ("row_start", row_start, i32, (n + 1,))])
        key = (code, n, max_rows, min(max_len, width * PAGE), heads)
        if self._need.get(key, self._ws_bytes + 1) > self._ws_bytes:
            self._workspace(key)
        self._call(self.lib.dflow_kv8_attention, code, self._ref, n, page_table.data_ptr(), width, kv_len.data_ptr(),
                   row_start.data_ptr(), rows, max_rows, max_len, heads, q.data_ptr(), ld_q,
                   self._scale if scale is None else scale, causal, out.data_ptr(), ld_o, self._ws_ptr, self._ws_bytes,
                   self._status)
        return out
