"""Python side of the page pool (include/kvc.h, ``kvc_pool_*``): answering from retained caches.

Argument marshalling only, as in ``binding``: every step runs in the CUDA library, PyTorch holds the memory and the
streams, and there is no CPU fallback.

    pool = Pool(32, 8, 128, torch.bfloat16, n_pages=4096, page_format="int8", n_layers=32, max_seqs=64)
    pool.write(layer, K[:, :n].transpose(0, 1), V[:, :n].transpose(0, 1), slots)   # a retained cache (Kvc.cache_view)
    plan = pool.plan([17, 250, 3])                                                 # three prompts, packed
    out, lse = pool.prompt(q, k, v, plan)
    out, lse = pool.decode(layer, q, table, lens, k, v)                            # one new token per sequence

A *slot* is ``page * page_size + row``; ``table`` holds a row of pages per sequence, ``lens`` how many rows it has.  All calls are
asynchronous on the current stream; what they find wrong on the device (a slot or page outside the pool, a length beyond the table)
is left out and reported by ``status()``.
"""
from __future__ import annotations

import ctypes
import dataclasses
from typing import Optional, Sequence, Tuple

import torch

from .binding import KVC_BF16, KVC_F32, KVC_OK, KVC_PAGES_INT8, KVC_PAGES_PLAIN, KvcError, KvcPoolConfig, KvcPromptPlan, _raw_stream, lib


@dataclasses.dataclass
class PromptPlan:
    """How a batch of packed prompts is cut into pieces of work; made once per batch, used by every layer."""

    plan: KvcPromptPlan
    items: torch.Tensor

    @property
    def n_tokens(self) -> int:
        return self.plan.n_tokens


class Pool:
    """A pool of key/value pages for many sequences, and attention over it.

    ``page_format`` "plain" holds ``dtype``, "int8" 8-bit codes with a scale per (token, kv-head).  ``blob`` may be a
    caller's own uint8 tensor [n_layers, Pool bytes per layer] instead of one allocated here.
    """

    def __init__(self, n_q_heads: int, n_kv_heads: int, head_dim: int, dtype: torch.dtype, n_pages: int, page_size: int = 64,
                 page_format: str = "plain", n_layers: int = 1, max_seqs: int = 256, softmax_scale: float = 0.0, device: int = 0,
                 blob: Optional[torch.Tensor] = None):
        if not torch.cuda.is_available():
            raise RuntimeError("kvc needs a CUDA device: there is no CPU implementation")
        self._lib = lib()
        self.dtype, self.device, self.head_dim = dtype, torch.device("cuda", device), head_dim
        self.n_q_heads, self.n_kv_heads, self.page_size, self.n_pages = n_q_heads, n_kv_heads, page_size, n_pages
        self.page_format, self._ordinal = page_format, device
        code = {torch.float32: KVC_F32, torch.bfloat16: KVC_BF16}[dtype]
        pages = {"plain": KVC_PAGES_PLAIN, "int8": KVC_PAGES_INT8}[page_format]
        cfg = KvcPoolConfig(n_q_heads, n_kv_heads, head_dim, code, pages, page_size, n_pages, max_seqs, softmax_scale, device, 0)
        h = ctypes.c_void_p()
        rc = self._lib.kvc_pool_create(ctypes.byref(cfg), ctypes.byref(h))
        if rc != KVC_OK:
            raise KvcError(rc, "kvc_pool_create rejected the configuration")
        self._h = h
        a, b = ctypes.c_size_t(), ctypes.c_size_t()
        self._check(self._lib.kvc_pool_nbytes(self._h, ctypes.byref(a), ctypes.byref(b)))
        self.blob_bytes, self.ws_bytes = a.value, b.value
        if blob is not None and (blob.dtype != torch.uint8 or blob.dim() != 2 or blob.stride(1) != 1 or blob.shape[1] < self.blob_bytes
                                 or blob.stride(0) % 256 and blob.shape[0] > 1 or blob.data_ptr() % 256 or blob.device != self.device):
            raise ValueError(f"blob: a uint8 tensor [layers, {self.blob_bytes}] on {self.device}, rows at multiples of 256 bytes")
        with torch.cuda.device(self.device):
            # (zeros: a page that was never written holds numbers, whatever reads it)
            self.blob = torch.zeros(n_layers, -(-self.blob_bytes // 256) * 256, dtype=torch.uint8, device=self.device) if blob is None else blob
            self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=self.device)
            self._ws = self.workspace.data_ptr()
            self.workspace_init()

    # -- helpers ---------------------------------------------------------------------------------
    def _layer(self, layer: int) -> int:
        blob = self.blob
        if not 0 <= layer < blob.shape[0]:
            raise IndexError(f"layer {layer} outside [0, {blob.shape[0]})")
        return blob.data_ptr() + layer * blob.stride(0)

    def _check(self, rc: int):
        if rc != KVC_OK:
            raise KvcError(rc, self._lib.kvc_pool_last_error(self._h).decode())

    def close(self):
        if getattr(self, "_h", None):
            self._lib.kvc_pool_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # (A call's host time is mostly these checks and the marshalling: one stride() for all three, get_device() instead of a comparison of
    # devices, new_empty() instead of empty(): decode 14 -> 10 us, write 8.6 -> 6.5.)
    def _rows(self, name: str, t: torch.Tensor, n: int, heads: int) -> Tuple[int, ...]:
        """The strides of rows [n][heads][d] of the pool's dtype; those of the first two dimensions are free."""
        st = t.stride()
        if t.dtype is not self.dtype or t.shape != (n, heads, self.head_dim) or t.get_device() != self._ordinal or (st[2] != 1 and t.numel()):
            raise ValueError(f"{name}: {self.dtype} rows [{n}, {heads}, {self.head_dim}] on {self.device}, innermost contiguous; got "
                             f"{t.dtype} {list(t.shape)} with strides {list(st)} on {t.device}")
        return st

    def _token_rows(self, name: str, t: torch.Tensor, n: int, heads: int) -> int:
        """The same with a token's heads side by side; the stride of a token's rows, in elements."""
        st = self._rows(name, t, n, heads)
        if st[1] != self.head_dim and heads > 1 and n:
            raise ValueError(f"{name}: the heads of a token must be contiguous, strides {list(st)}")
        return st[0] if n > 1 else max(st[0], heads * self.head_dim)

    def _index(self, name: str, t: torch.Tensor, dtype: torch.dtype) -> int:
        if t.dtype is not dtype or t.get_device() != self._ordinal or not t.is_contiguous():
            raise ValueError(f"{name}: a contiguous {dtype} tensor on {self.device}; got {t.dtype} on {t.device}")
        return t.data_ptr()

    def _pair_strides(self, k: torch.Tensor, v: torch.Tensor, n: int) -> Tuple[int, int]:
        """Strides (token, kv-head) of two row tensors, which must agree; dimensions of one element may say anything."""
        heads, d = self.n_kv_heads, self.head_dim
        a, b = self._rows("k", k, n, heads), self._rows("v", v, n, heads)
        if a != b and (n > 1 and a[0] != b[0] or heads > 1 and a[1] != b[1]):
            raise ValueError(f"k and v must have the same strides; got {list(a)} and {list(b)}")
        return (a[0] if n > 1 else d), (a[1] if heads > 1 else d)

    # -- pages -----------------------------------------------------------------------------------
    def slots(self, pages: torch.Tensor, n: int, first: int = 0) -> torch.Tensor:
        """int64 [n]: the slots of rows first .. first + n - 1 of a sequence whose pages (a row of a table) are given."""
        at = torch.arange(first, first + n, device=pages.device)
        return pages.long()[at // self.page_size] * self.page_size + at % self.page_size

    def pages(self, layer: int) -> Tuple[torch.Tensor, ...]:
        """(K, V) or (K codes, V codes, K scales, V scales) of a layer, aliasing the blob: [page][kv-head][row]([d])."""
        held = (self.n_pages, self.n_kv_heads, self.page_size, self.head_dim)
        rows = self.n_pages * self.n_kv_heads * self.page_size
        blob = self.blob[layer]
        if self.page_format == "plain":
            size = rows * self.head_dim * self.dtype.itemsize
            return tuple(blob[i * size:(i + 1) * size].view(self.dtype).view(held) for i in (0, 1))
        size, up = rows * self.head_dim, -(-rows * 4 // 256) * 256
        return tuple(blob[i * size:(i + 1) * size].view(torch.int8).view(held) for i in (0, 1)) + \
            tuple(blob[2 * size + i * up:][:rows * 4].view(torch.float32).view(held[:3]) for i in (0, 1))

    def write(self, layer: int, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor) -> None:
        """Rows k, v [n][Hkv][d] (any strides of the first two dimensions, the same for both) into ``slots`` int64 [n]."""
        n = slots.shape[0]
        ts, hs = self._pair_strides(k, v, n)
        rc = self._lib.kvc_pool_write(self._h, k.data_ptr(), v.data_ptr(), ts, hs, self._index("slots", slots, torch.int64), n,
                                      self._layer(layer), self._ws, _raw_stream(self._ordinal))
        if rc:
            self._check(rc)

    def read(self, layer: int, slots: torch.Tensor, k: Optional[torch.Tensor] = None,
             v: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """Slots back as rows [n][Hkv][d] of the pool's dtype, into k and v if given."""
        n = slots.shape[0]
        if (k is None) != (v is None):
            raise ValueError("k and v go together")
        if k is None:
            shape = (n, self.n_kv_heads, self.head_dim)
            at = self._index("slots", slots, torch.int64)
            k, v = slots.new_empty(shape, dtype=self.dtype), slots.new_empty(shape, dtype=self.dtype)
            ts, hs = self.n_kv_heads * self.head_dim, self.head_dim
        else:
            at = self._index("slots", slots, torch.int64)
            ts, hs = self._pair_strides(k, v, n)
        rc = self._lib.kvc_pool_read(self._h, self._layer(layer), at, n, k.data_ptr(), v.data_ptr(), ts, hs, self._ws, _raw_stream(self._ordinal))
        if rc:
            self._check(rc)
        return k, v

    # -- attention -------------------------------------------------------------------------------
    def _results(self, q: torch.Tensor, n: int, out: Optional[torch.Tensor], lse: Optional[torch.Tensor]) -> Tuple[torch.Tensor, torch.Tensor]:
        heads = self.n_q_heads
        if out is None:
            out = q.new_empty((n, heads, self.head_dim))
        else:
            self._rows("out", out, n, heads)
            if not out.is_contiguous():
                raise ValueError("out must be contiguous")
        if lse is None:
            lse = q.new_empty((n, heads), dtype=torch.float32)
        else:
            self._index("lse", lse, torch.float32)
            if lse.shape != (n, heads):
                raise ValueError(f"lse: [{n}, {heads}]; got {list(lse.shape)}")
        return out, lse

    def decode(self, layer: int, q: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, k: Optional[torch.Tensor] = None,
               v: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
               lse: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """(out [n][Hq][d], lse [n][Hq]) of one new token per sequence: q [n][Hq][d], table int32 [n][pages], lens int32 [n].

        With k, v [n][Hkv][d] the token's own row is written to row ``lens[i]`` of its sequence and takes part; ``lens`` stays as
        it is (the caller adds one when all layers are done).
        """
        n = q.shape[0]
        q_stride = self._token_rows("q", q, n, self.n_q_heads)
        if len(pages := table.shape) != 2 or pages[0] != n or lens.shape != (n,):
            raise ValueError(f"table [{n}, pages] and lens [{n}]; got {list(table.shape)} and {list(lens.shape)}")
        if (k is None) != (v is None):
            raise ValueError("k and v go together")
        kv_stride, kp, vp = 0, None, None
        if k is not None:
            kv_stride = self._token_rows("k", k, n, self.n_kv_heads)
            if self._token_rows("v", v, n, self.n_kv_heads) != kv_stride:
                raise ValueError(f"k and v must have the same strides; got {list(k.stride())} and {list(v.stride())}")
            kp, vp = k.data_ptr(), v.data_ptr()
        out, lse = self._results(q, n, out, lse)
        rc = self._lib.kvc_pool_decode(self._h, q.data_ptr(), q_stride, kp, vp, kv_stride, self._index("table", table, torch.int32),
                                       pages[1], self._index("lens", lens, torch.int32), n, self._layer(layer), self._ws,
                                       out.data_ptr(), lse.data_ptr(), _raw_stream(self._ordinal))
        if rc:
            self._check(rc)
        return out, lse

    def plan(self, lens: Sequence[int]) -> PromptPlan:
        """The plan of prompts of these lengths (host numbers), packed in this order."""
        lens = [int(x) for x in lens]
        if any(not -2 ** 31 <= x < 2 ** 31 for x in lens):
            raise ValueError("lengths are 32-bit numbers")
        arr = (ctypes.c_int * len(lens))(*lens)
        plan = KvcPromptPlan()
        self._check(self._lib.kvc_pool_plan(self._h, arr, len(lens), ctypes.byref(plan), None))
        items = torch.empty(plan.item_bytes, dtype=torch.uint8)
        self._check(self._lib.kvc_pool_plan(self._h, arr, len(lens), ctypes.byref(plan), items.data_ptr() if plan.item_bytes else None))
        return PromptPlan(plan, items.to(self.device))

    def prompt(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, plan: PromptPlan, out: Optional[torch.Tensor] = None,
               lse: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """(out [N][Hq][d], lse [N][Hq]) of packed prompts q [N][Hq][d], k, v [N][Hkv][d], causal inside each."""
        n = plan.plan.n_tokens
        q_stride = self._token_rows("q", q, n, self.n_q_heads)
        kv_stride = self._token_rows("k", k, n, self.n_kv_heads)
        if self._token_rows("v", v, n, self.n_kv_heads) != kv_stride:
            raise ValueError(f"k and v must have the same strides; got {list(k.stride())} and {list(v.stride())}")
        out, lse = self._results(q, n, out, lse)
        rc = self._lib.kvc_pool_prompt(self._h, q.data_ptr(), q_stride, k.data_ptr(), v.data_ptr(), kv_stride, ctypes.byref(plan.plan),
                                       plan.items.data_ptr(), self._ws, out.data_ptr(), lse.data_ptr(), _raw_stream(self._ordinal))
        if rc:
            self._check(rc)
        return out, lse

    # -- state -----------------------------------------------------------------------------------
    def workspace_init(self) -> None:
        self._check(self._lib.kvc_pool_workspace_init(self._h, self._ws, _raw_stream(self._ordinal)))

    def status(self) -> int:
        return self._lib.kvc_pool_status(self._h, self._ws, _raw_stream(self._ordinal))

    def launch_count(self) -> int:
        return self._lib.kvc_pool_launch_count(self._h)

    def last_error(self) -> str:
        return self._lib.kvc_pool_last_error(self._h).decode()
