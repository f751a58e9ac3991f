"""Paged KV cache in 8 bits: page tables sized to the requests (PagePool), the
append of key and value rows and the attention over them (KV8Cache).

Argument marshalling over dflow_page_resize, dflow_kv8_append and
dflow_kv8_attention; the layouts are theirs (include/dflow.h).  The tensors
belong to the caller and every call is asynchronous on torch's current stream
of their device.  Calls through one KV8Cache share its workspace, so they must
execute in order: one stream, or streams ordered by events; graphs captured
through one cache are replayed one at a time.  What only the device can see
(a page id outside the pool, a sequence that does not fit) sets bits of the
object's status word, which status() reads.
"""
from __future__ import annotations

import contextlib
import ctypes
import math
from typing import Optional

from .runtime import DFLOW_BF16, DFLOW_F32, KV8, PAGE, DFlowError, Pool, load_library

GROUP = 16                     # tokens per scale
WORKSPACE_ZEROED = 4096        # DFLOW_KV8_WORKSPACE_ZEROED


def _same_device(dev, **tensors):
    for name, t in tensors.items():
        if t is not None and t.device != dev:
            raise DFlowError(f"{name} is on {t.device}, not on {dev}")


def _check_i32(torch, name, t, shape):
    if t.dtype is not torch.int32 or t.dim() != len(shape) or not t.is_contiguous():
        raise DFlowError(f"{name} must be a contiguous int32 tensor of {len(shape)} dimension(s)")
    for have, want in zip(t.shape, shape):
        if want is not None and have < want:
            raise DFlowError(f"{name} has shape {tuple(t.shape)}, at least {shape} needed")


class _DeviceCalls:
    """Library calls on a device's current stream, with a status word."""

    def _open(self, t):
        import torch
        if t.device.type != "cuda":
            raise DFlowError("the 8-bit cache needs a HIP device; there is no CPU path")
        self.torch, self.device, self.lib = torch, t.device, load_library()
        self.status_word = torch.zeros(1, dtype=torch.int32, device=t.device)
        self._status = self.status_word.data_ptr()

    def _on(self):
        """The device of the tensors made current (usually it is)."""
        cuda = self.torch.cuda
        return contextlib.nullcontext() if cuda.current_device() == self.device.index else cuda.device(self.device)

    def _stream(self):
        return self.torch.cuda.current_stream(self.device).cuda_stream

    def _check(self, rc: int, what: str):
        if rc != 0:
            raise DFlowError(f"{what} failed ({rc}): {self.lib.dflow_last_error().decode()}")

    def status(self, clear: bool = True) -> int:
        """DFLOW_STATUS_* bits set by the calls so far (waits for the current stream)."""
        with self._on():
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
        torch = self.torch
        _same_device(self.device, n_held=n_held, free_pages=free_pages, n_free=n_free)
        _check_i32(torch, "page_table", page_table, (1, 1))
        _check_i32(torch, "n_held", n_held, (page_table.shape[0],))
        _check_i32(torch, "free_pages", free_pages, (1,))
        _check_i32(torch, "n_free", n_free, (1,))
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
        torch, n = self.torch, seq_len.shape[0]
        _same_device(self.device, seq_len=seq_len, new_len=new_len, slot=slot, row_start=row_start)
        _check_i32(torch, "seq_len", seq_len, (1,))
        if n > self.page_table.shape[0]:
            raise DFlowError(f"{n} sequences, {self.page_table.shape[0]} page-table rows")
        if new_len is not None:
            _check_i32(torch, "new_len", new_len, (n,))
        if slot is not None:
            if new_len is None or row_start is None:
                raise DFlowError("a slot map needs new_len and row_start")
            _check_i32(torch, "slot", slot, (None,))
            _check_i32(torch, "row_start", row_start, (n + 1,))
        p = lambda t: None if t is None else t.data_ptr()
        with self._on():
            self._check(self.lib.dflow_page_resize(
                self._stream(), self._ref, n, seq_len.data_ptr(), p(new_len), p(slot),
                0 if slot is None else slot.shape[0], p(row_start), self._status), "dflow_page_resize")


class KV8Cache(_DeviceCalls):
    """One layer's 8-bit cache: k uint8 [num_pages, n_kv_heads, 64, head_dim],
    v uint8 [num_pages, n_kv_heads, head_dim, 64] (e4m3 codes), k_scale and
    v_scale fp32 [num_pages, n_kv_heads, 4]."""

    def __init__(self, k, v, k_scale, v_scale):
        self._open(k)
        torch = self.torch
        _same_device(self.device, v=v, k_scale=k_scale, v_scale=v_scale)
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
        self._ws, self._ws_bytes, self._kept = None, 0, []
        self._need = {}

    @classmethod
    def alloc(cls, num_pages: int, n_kv_heads: int, head_dim: int, device="cuda:0") -> "KV8Cache":
        """A cache of zeros with unit scales."""
        import torch
        u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8, device=device)
        one = lambda: torch.ones(num_pages, n_kv_heads, PAGE // GROUP, dtype=torch.float32, device=device)
        return cls(u8(num_pages, n_kv_heads, PAGE, head_dim), u8(num_pages, n_kv_heads, head_dim, PAGE), one(), one())

    def _rows(self, name, t, heads):
        """(dtype code, row stride in elements) of a [rows, heads, head_dim] tensor whose rows are dense."""
        code = self._codes.get(t.dtype)
        if code is None:
            raise DFlowError(f"{name} must be bfloat16 or float32, got {t.dtype}")
        n, h, d = t.shape if t.dim() == 3 else (0, 0, 0)
        if d != self.head_dim or (heads is not None and h != heads) or h < 1:
            raise DFlowError(f"{name} has shape {tuple(t.shape)}, [rows, {heads or 'heads'}, {self.head_dim}] needed")
        s = t.stride()
        if s[2] != 1 or (h > 1 and s[1] != d):
            raise DFlowError(f"{name}: the heads of a row must be contiguous (strides {s})")
        return code, (s[0] if n > 1 else h * d)

    def append(self, k, v, slot):
        """dflow_kv8_append: rows k, v [rows, n_kv_heads, head_dim] (bf16 or fp32) to their slots (int32 [rows], -1: none)."""
        dev, n = self.device, k.shape[0]
        if k.device != dev or v.device != dev or slot.device != dev:
            _same_device(dev, k=k, v=v, slot=slot)
        code, ld_k = self._rows("k", k, self.n_kv_heads)
        code_v, ld_v = self._rows("v", v, self.n_kv_heads)
        if code_v != code or v.shape[0] != n:
            raise DFlowError(f"k {k.dtype} {tuple(k.shape)} and v {v.dtype} {tuple(v.shape)} differ")
        _check_i32(self.torch, "slot", slot, (n,))
        with self._on():
            self._check(self.lib.dflow_kv8_append(self._stream(), code, self._ref, n, k.data_ptr(), ld_k, v.data_ptr(),
                                                  ld_v, slot.data_ptr(), self._status), "dflow_kv8_append")

    def _workspace(self, key):
        """Workspace for calls of these sizes.  A buffer that is outgrown is kept: graphs captured with it hold its address."""
        need = self._need.get(key)
        if need is None:
            need = self.lib.dflow_kv8_attention_workspace(*key, self.n_kv_heads, self.head_dim)
            if need == ctypes.c_size_t(-1).value:
                self._check(-1, "dflow_kv8_attention_workspace")
            if len(self._need) >= 4096:
                self._need.clear()
            self._need[key] = need
        if need > self._ws_bytes:
            if self._ws is not None:
                self._kept.append(self._ws)
            self._ws_bytes = max(need, 2 * self._ws_bytes)
            self._ws = self.torch.empty(self._ws_bytes, dtype=self.torch.uint8, device=self.device)
            self._ws[:WORKSPACE_ZEROED].zero_()

    def attention(self, q, page_table, kv_len, row_start, max_rows: int, max_len: int, causal: bool = True,
                  scale: Optional[float] = None, out=None):
        """dflow_kv8_attention: q [rows, n_heads, head_dim] (bf16 or fp32) of
        len(kv_len) sequences, rows row_start[s] .. row_start[s + 1] - 1 each, over
        kv_len[s] cached tokens.  max_rows and max_len bound both.  scale
        defaults to head_dim^-1/2.  Returns out."""
        torch, dev, n = self.torch, self.device, kv_len.shape[0]
        if out is None:
            out = torch.zeros(q.shape, dtype=q.dtype, device=q.device)
        _same_device(dev, q=q, page_table=page_table, kv_len=kv_len, row_start=row_start, out=out)
        code, ld_q = self._rows("q", q, None)
        code_o, ld_o = self._rows("out", out, q.shape[1])
        if code_o != code or out.shape != q.shape:
            raise DFlowError(f"q {q.dtype} {tuple(q.shape)} and out {out.dtype} {tuple(out.shape)} differ")
        _check_i32(torch, "page_table", page_table, (n, 1))
        _check_i32(torch, "kv_len", kv_len, (1,))
        _check_i32(torch, "row_start", row_start, (n + 1,))
        max_pages = page_table.shape[1]
        with self._on():
            self._workspace((code, n, max_rows, min(max_len, max_pages * PAGE), q.shape[1]))
            self._check(self.lib.dflow_kv8_attention(
                self._stream(), code, self._ref, n, page_table.data_ptr(), max_pages, kv_len.data_ptr(),
                row_start.data_ptr(), q.shape[0], max_rows, max_len, q.shape[1], q.data_ptr(), ld_q,
                self._scale if scale is None else scale, bool(causal), out.data_ptr(), ld_o,
                None if self._ws is None else self._ws.data_ptr(), self._ws_bytes, self._status),
                "dflow_kv8_attention")
        return out
