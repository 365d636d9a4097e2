"""GB300-native bounded KV-cache recomputation (CacheReforge, arXiv 2609.30884).

Python binding of the C ABI in include/crf.h. Objects here hold the caller's
torch tensors and the ctypes structs that point into them; the calls marshal
pointers, sizes and the current CUDA stream into libcrf.so. Nothing in this
package computes any step of the path.

    ctx = Context(0)
    model = Model(dims, layers, embed, final_norm, lm_head)
    cur = Adapter(lora, layers)                      # {module: (A, B)} per layer
    pool = KVPool(k_pages, v_pages)                  # per-layer [P, Hkv, 16, d] bf16
    req = Request(page_table, s, e, tokens=..., hidden_in=..., hidden_out=[...],
                  final_hidden_out=...)
    ws = ctx.workspace(model, cur, [req])
    ctx.recompute_window(model, cur, pool, [req], ws)
    ctx.drift(model.dims_c, cur, anchors, out_sq, ctx.drift_workspace(...))
    ctx.kl(model, ref_hidden, cur_hidden, out_kl, ...)

A recovered cache is extended with new tokens by calls of one layer and of the pool's pages:

    rope = Rope(head_dim, theta=1e6)
    chunks = Chunks(page_tables, n_new, pos)         # one for all layers of a step
    ctx.cache_append(pool, layer, chunks, k, v, q=q, q_out=q_rot, rope=rope)
    ctx.chunk_attention(pool, layer, chunks, q_rot, o, ctx.chunk_attention_workspace(pool, chunks, n_heads))
    ctx.pages_fork(pool, refs, PageTables(tables, n_tokens, child_tables), ctx.pages_workspace(...))
"""
from __future__ import annotations

import ctypes
import struct
from ctypes import POINTER, byref, c_size_t, c_void_p
from typing import Dict, List, Optional, Sequence, Tuple

import torch

from . import abi
from .abi import CrfError

MODULES = ("q", "k", "v", "o", "gate", "up", "down")

__all__ = ["Context", "Model", "Adapter", "KVPool", "Request", "Rope", "Chunks", "PageTables", "CrfError",
           "MODULES", "abi", "kl_logits_noalloc"]


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


class Model:
    """Base model: dims plus per-layer weight tensors (bf16 on the device)."""

    def __init__(self, dims: dict, layers: Sequence[Dict[str, torch.Tensor]],
                 embed: Optional[torch.Tensor] = None, final_norm: Optional[torch.Tensor] = None,
                 lm_head: Optional[torch.Tensor] = None):
        self.tensors = (list(layers), embed, final_norm, lm_head)
        self.dims = dict(dims)
        self.dims_c = abi.ModelDims(dims["n_layers"], dims["hidden"], dims["n_q_heads"],
                                    dims["n_kv_heads"], dims["head_dim"], dims["ffn"],
                                    dims["vocab"], dims["rms_eps"], dims["rope_theta"],
                                    int(bool(dims["qkv_bias"])))
        n = dims["n_layers"]
        self._layers = (abi.LayerWeights * n)()
        for l, w in enumerate(layers):
            if w is None:
                continue
            lw = self._layers[l]
            for j, m in enumerate(MODULES):
                lw.W[j] = _ptr(w.get(f"W_{m}"))
            for j, m in enumerate(("q", "k", "v")):
                lw.bias[j] = _ptr(w.get(f"bias_{m}"))
            lw.ln1 = _ptr(w.get("ln1"))
            lw.ln2 = _ptr(w.get("ln2"))
        self.c = abi.Model(self.dims_c, self._layers, _ptr(embed), _ptr(final_norm), _ptr(lm_head))


class Adapter:
    """One adapter version: per-layer {module: (A [r, in], B [out, r])} bf16 device tensors."""

    def __init__(self, rank: int, alpha: float, modules: Sequence[str],
                 layers: Sequence[Optional[Dict[str, Tuple[torch.Tensor, torch.Tensor]]]]):
        self.layers = list(layers)
        mask = sum(1 << MODULES.index(m) for m in modules)
        n = len(layers)
        self._A = (c_void_p * (n * 7))()
        self._B = (c_void_p * (n * 7))()
        for l, d in enumerate(layers):
            if d is None:
                continue
            for m, (A, B) in d.items():
                j = MODULES.index(m)
                self._A[l * 7 + j] = A.data_ptr()
                self._B[l * 7 + j] = B.data_ptr()
        self.dims_c = abi.LoraDims(rank, alpha, mask)
        self.c = abi.Adapter(self.dims_c, self._A, self._B)


class KVPool:
    """Per-layer K and V page pools, bf16 [num_pages, Hkv, 16, d]. Calls that are given the model take flat views
    of that memory too; those that extend a cache read the heads and their size from the shape."""

    def __init__(self, k_pages: Sequence[torch.Tensor], v_pages: Sequence[torch.Tensor]):
        self.k_pages, self.v_pages = list(k_pages), list(v_pages)
        n = len(self.k_pages)
        self._k = (c_void_p * n)(*[t.data_ptr() for t in self.k_pages])
        self._v = (c_void_p * n)(*[t.data_ptr() for t in self.v_pages])
        shape = [int(x) for x in self.k_pages[0].shape]
        self.num_pages = shape[0]
        self.n_kv_heads, self.head_dim = (shape[1], shape[3]) if len(shape) == 4 else (None, None)
        self.device = self.k_pages[0].get_device()
        self.not_paged = self._not_paged(shape)
        self.c = abi.KVPool(self._k, self._v, self.num_pages)
        self.address = ctypes.addressof(self.c)

    def _not_paged(self, shape: List[int]) -> Optional[str]:
        """Why the tensors do not all hold ``shape[0]`` pages of layer 0's keys' shape, or None: the calls that extend a
        cache write by that shape alone."""
        if len(shape) != 4 or shape[2] != abi.PAGE_SIZE:
            return f"the pool's tensors must be [num_pages, kv heads, {abi.PAGE_SIZE}, head_dim]"
        if len(self.v_pages) != len(self.k_pages):
            return "the pool has a different number of K and V layers"
        for name, layers in (("k_pages", self.k_pages), ("v_pages", self.v_pages)):
            for l, t in enumerate(layers):
                if t.dtype != torch.bfloat16 or t.device != self.k_pages[0].device or not t.is_contiguous():
                    return f"{name}[{l}] must be contiguous bfloat16 on the device of k_pages[0]"
                if t.dim() != 4 or list(t.shape[1:]) != shape[1:] or t.shape[0] < shape[0]:
                    return f"{name}[{l}] must hold {shape[0]} pages {shape[1:]} like k_pages[0], not {list(t.shape)}"
        return None


class Request:
    """One cached prefix and the window [s, e) to refresh (see crf_request)."""

    def __init__(self, page_table: torch.Tensor, s: int, e: int, n_tokens: Optional[int] = None,
                 tokens: Optional[torch.Tensor] = None, hidden_in: Optional[torch.Tensor] = None,
                 hidden_out: Optional[Sequence[torch.Tensor]] = None,
                 final_hidden_out: Optional[torch.Tensor] = None):
        if n_tokens is None:
            n_tokens = int(tokens.shape[0]) if tokens is not None else int(hidden_in.shape[0])
        self.keep = (page_table, tokens, hidden_in, hidden_out, final_hidden_out)
        self._hout = None
        if hidden_out is not None:
            self._hout = (c_void_p * max(1, len(hidden_out)))(*[t.data_ptr() for t in hidden_out])
        self.c = abi.Request(n_tokens, s, e, page_table.data_ptr(), _ptr(tokens), _ptr(hidden_in),
                             self._hout, _ptr(final_hidden_out))


_INT32 = 1 << 31  # ctypes drops the bits of an int that its field has no room for


def _fits(name: str, v: int) -> int:
    if not -_INT32 <= v < _INT32:
        raise ValueError(f"{name} {v} does not fit 32 bits")
    return v


class Rope:
    """Rotary positions (see crf_rope): the first ``rot_dim`` elements of a head turn in pairs of ``layout``
    ("half" or "interleaved"); ``scaling`` "none", "linear", "base" or "bands" for contexts ``factor`` times
    as long. "bands" ramps over the turns that a pair makes in ``original`` positions, not over its index."""

    def __init__(self, head_dim: int, rot_dim: Optional[int] = None, theta: float = 1e4, layout: str = "half",
                 scaling: str = "none", factor: float = 1.0, low: float = 1.0, high: float = 32.0,
                 original: float = 4096.0, magnitude: float = 1.0):
        if layout not in abi.ROPE_LAYOUTS:
            raise ValueError(f"layout must be one of {sorted(abi.ROPE_LAYOUTS)}")
        if scaling not in abi.ROPE_SCALINGS:
            raise ValueError(f"scaling must be one of {sorted(abi.ROPE_SCALINGS)}")
        self.head_dim = _fits("head_dim", head_dim)
        self.c = abi.Rope(head_dim, head_dim if rot_dim is None else _fits("rot_dim", rot_dim), abi.ROPE_LAYOUTS[layout],
                          abi.ROPE_SCALINGS[scaling], theta, factor, low, high, original, magnitude)
        self.address = ctypes.addressof(self.c)


def _int32_on_device(name: str, t: torch.Tensor, n: int) -> torch.Tensor:
    if t.dtype != torch.int32 or not t.is_contiguous() or t.numel() < n:
        raise ValueError(f"{name} must be a contiguous int32 tensor of at least {n} entries")
    return t


def _one_device(tensors: Sequence[torch.Tensor]) -> int:
    devices = {t.get_device() for t in tensors}
    if len(devices) > 1:
        raise ValueError("the page tables are on different devices")
    return devices.pop() if devices else -1


class Chunks:
    """The new rows of a step's requests (see crf_chunk), packed in order: ``n_new[i]`` rows at positions
    ``pos[i]`` on of the request cached on ``page_tables[i]``. ``n_keys[i]`` (default ``pos + n_new``)
    cached positions are there for attention to see. One object serves every layer of a step."""

    def __init__(self, page_tables: Sequence[torch.Tensor], n_new: Sequence[int], pos: Sequence[int],
                 n_keys: Optional[Sequence[int]] = None):
        n = len(page_tables)
        if len(n_new) != n or len(pos) != n or (n_keys is not None and len(n_keys) != n):
            raise ValueError("page_tables, n_new, pos and n_keys must have one entry a request")
        self.page_tables = list(page_tables)
        self.n, self.rows = n, sum(n_new)
        self.device = _one_device(self.page_tables)
        self.append_entries, self.attend_entries = [], []
        self.c = (abi.Chunk * max(1, n))()
        for i, t in enumerate(self.page_tables):
            m, p = int(n_new[i]), int(pos[i])
            k = p + m if n_keys is None else int(n_keys[i])
            if not (-_INT32 <= m < _INT32 and -_INT32 <= p < _INT32 and -_INT32 <= k < _INT32):
                raise ValueError(f"request {i}: n_new, pos or n_keys does not fit 32 bits")
            if t.dtype != torch.int32 or not t.is_contiguous():
                raise ValueError(f"page table {i} must be a contiguous int32 tensor")
            self.append_entries.append((p + m + 15) // 16 if m else 0)
            self.attend_entries.append((k + 15) // 16 if m else 0)
            self.c[i] = abi.Chunk(m, p, k, t.data_ptr())
        self.address = ctypes.addressof(self.c)
        self.append_ok = all(t.numel() >= e for t, e in zip(self.page_tables, self.append_entries))
        self.attend_ok = all(t.numel() >= e for t, e in zip(self.page_tables, self.attend_entries))


class PageTables:
    """Page tables of requests of ``n_tokens[i]`` tokens for the pages_* calls (see crf_pages); ``outs``
    receives the new tables."""

    def __init__(self, tables: Sequence[torch.Tensor], n_tokens: Sequence[int],
                 outs: Optional[Sequence[torch.Tensor]] = None):
        n = len(tables)
        if len(n_tokens) != n or (outs is not None and len(outs) != n):
            raise ValueError("tables, n_tokens and outs must have one entry a request")
        self.tables, self.outs = list(tables), None if outs is None else list(outs)
        self.device = _one_device(self.tables + (self.outs or []))
        self.n = n
        self.c = (abi.Pages * max(1, n))()
        for i, t in enumerate(self.tables):
            count = int(n_tokens[i])
            if not -_INT32 <= count < _INT32:
                raise ValueError(f"table {i}: n_tokens does not fit 32 bits")
            need = (count + 15) // 16
            _int32_on_device(f"table {i}", t, need)
            if outs is not None:
                _int32_on_device(f"outs[{i}]", outs[i], need)
            self.c[i] = abi.Pages(count, t.data_ptr(), None if outs is None else outs[i].data_ptr())
        self.address = ctypes.addressof(self.c)


_TYPES = {torch.bfloat16: abi.BF16, torch.float16: abi.FP16, torch.float32: abi.FP32}
# The current stream's handle: a torch.cuda.Stream object costs a small call as much as half its launch.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda d: torch.cuda.current_stream(d).cuda_stream)
# crf_heads, packed into a context's buffer: building the ctypes structures takes three times as long.
_pack_heads = struct.Struct("PPiqqqq").pack_into
_HEADS = ctypes.sizeof(abi.Heads)


def _put_heads(buf, at: int, device: int, name: str, x: torch.Tensor, out: Optional[torch.Tensor], dim: int) -> int:
    """crf_heads of x [rows, heads, dim] and out (any row and head strides) at ``buf[at:]``; the heads."""
    shape = x.shape
    if len(shape) != 3 or shape[2] != dim:
        raise ValueError(f"{name} must be [rows, heads, {dim}]")
    if x.get_device() != device:
        raise ValueError(f"{name} must be on cuda:{device}")
    row, head, one = x.stride()
    if out is None:
        _pack_heads(buf, at, x.data_ptr(), 0, shape[1], row, head, 0, 0)
    elif out is x:
        p = x.data_ptr()
        _pack_heads(buf, at, p, p, shape[1], row, head, row, head)
    else:
        if out.shape != shape or out.dtype != x.dtype or out.get_device() != device:
            raise ValueError(f"{name}: the output must have the input's shape, type and device")
        out_row, out_head, out_one = out.stride()
        if out_one != 1:
            raise ValueError(f"{name}: the elements of a head must be adjacent")
        _pack_heads(buf, at, x.data_ptr(), out.data_ptr(), shape[1], row, head, out_row, out_head)
    if one != 1:
        raise ValueError(f"{name}: the elements of a head must be adjacent")
    return shape[1]


def _req_array(reqs: Sequence[Request]):
    arr = (abi.Request * len(reqs))()
    for i, r in enumerate(reqs):
        arr[i] = r.c
    return arr


class Context:
    """A library context on one CUDA device."""

    def __init__(self, device: int = 0):
        self.lib = abi.load()
        self.device = device
        h = c_void_p()
        abi.check(self.lib.crf_create(byref(h), device))
        self.h = h
        self._parts = ctypes.create_string_buffer(3 * _HEADS)

    def close(self) -> None:
        if self.h:
            self.lib.crf_destroy(self.h)
            self.h = c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -------------------------------------------------------------- window
    def workspace_size(self, model: Model, adapter: Adapter, reqs: Sequence[Request]) -> int:
        n = c_size_t()
        arr = _req_array(reqs)
        abi.check(self.lib.crf_workspace_size(self.h, byref(model.c), byref(adapter.dims_c), arr,
                                              len(reqs), byref(n)))
        return n.value

    def workspace(self, model: Model, adapter: Adapter, reqs: Sequence[Request]) -> torch.Tensor:
        return torch.empty(max(256, self.workspace_size(model, adapter, reqs)), dtype=torch.uint8,
                           device=f"cuda:{self.device}")

    def recompute_window(self, model: Model, adapter: Adapter, pool: KVPool,
                         reqs: Sequence[Request], workspace: torch.Tensor, stream=None) -> None:
        arr = _req_array(reqs)
        abi.check(self.lib.crf_recompute_window(self.h, byref(model.c), byref(adapter.c),
                                                byref(pool.c), arr, len(reqs),
                                                workspace.data_ptr(), workspace.numel(),
                                                _stream(stream)))

    # -------------------------------------------------------------- generation
    @staticmethod
    def _decode_rows(positions: Sequence[int], page_tables: Sequence[torch.Tensor],
                     tokens: torch.Tensor):
        n = len(positions)
        arr = (abi.DecodeRow * n)()
        for i in range(n):
            arr[i] = abi.DecodeRow(int(positions[i]), page_tables[i].data_ptr(), tokens[i:i + 1].data_ptr())
        return arr

    def decode_workspace(self, model: Model, adapter: Adapter, positions: Sequence[int],
                         page_tables: Sequence[torch.Tensor], tokens: torch.Tensor) -> torch.Tensor:
        n = c_size_t()
        arr = self._decode_rows(positions, page_tables, tokens)
        abi.check(self.lib.crf_decode_workspace_size(self.h, byref(model.c), byref(adapter.dims_c), arr,
                                                     len(positions), byref(n)))
        return torch.empty(max(256, n.value), dtype=torch.uint8, device=f"cuda:{self.device}")

    def decode_step(self, model: Model, adapter: Adapter, pool: KVPool, positions: Sequence[int],
                    page_tables: Sequence[torch.Tensor], tokens: torch.Tensor, next_tokens: torch.Tensor,
                    workspace: torch.Tensor, logits: Optional[torch.Tensor] = None, stream=None) -> None:
        """One generated token per row: tokens[i] (device int32) sits at positions[i]; its K/V are
        written into the row's pages and next_tokens[i] receives the greedy next token."""
        arr = self._decode_rows(positions, page_tables, tokens)
        abi.check(self.lib.crf_decode_step(self.h, byref(model.c), byref(adapter.c), byref(pool.c), arr,
                                           len(positions), next_tokens.data_ptr(), _ptr(logits),
                                           workspace.data_ptr(), workspace.numel(), _stream(stream)))

    # -------------------------------------------------------------- drift
    def drift_workspace(self, dims_c, lora_dims_c) -> torch.Tensor:
        n = c_size_t()
        abi.check(self.lib.crf_drift_workspace_size(self.h, byref(dims_c), byref(lora_dims_c),
                                                    byref(n)))
        return torch.empty(max(256, n.value), dtype=torch.uint8, device=f"cuda:{self.device}")

    def drift(self, dims_c, cur: Adapter, anchors: Sequence[Adapter], out_sq: torch.Tensor,
              workspace: torch.Tensor, stream=None) -> None:
        arr = (POINTER(abi.Adapter) * len(anchors))(*[ctypes.pointer(a.c) for a in anchors])
        abi.check(self.lib.crf_drift(self.h, byref(dims_c), byref(cur.c), arr, out_sq.data_ptr(),
                                     workspace.data_ptr(), workspace.numel(), _stream(stream)))

    # -------------------------------------------------------------- KL
    def kl_workspace(self, n_rows: int, vocab: int, hidden: int = 0) -> torch.Tensor:
        n = c_size_t()
        abi.check(self.lib.crf_kl_workspace_size(self.h, n_rows, vocab, hidden, byref(n)))
        return torch.empty(max(256, n.value), dtype=torch.uint8, device=f"cuda:{self.device}")

    def kl(self, model: Optional[Model], ref: torch.Tensor, cur: torch.Tensor, out_kl: torch.Tensor,
           vocab: int, workspace: torch.Tensor, logits_out: Optional[torch.Tensor] = None,
           stream=None) -> None:
        abi.check(self.lib.crf_kl(self.h, byref(model.c) if model is not None else None,
                                  ref.data_ptr(), cur.data_ptr(), int(ref.shape[0]), vocab,
                                  out_kl.data_ptr(), _ptr(logits_out), workspace.data_ptr(),
                                  workspace.numel(), _stream(stream)))

    # -------------------------------------------------------------- extension by new tokens
    def _stream_here(self, stream) -> int:
        return _raw_stream(self.device) if stream is None else _stream(stream)

    def _here(self, *tensors: Optional[torch.Tensor]) -> None:
        device = self.device
        for t in tensors:
            if t is not None and t.get_device() != device:
                raise ValueError(f"every tensor of the call must be on cuda:{device}")

    def rotary(self, rope: Rope, positions: torch.Tensor, x: torch.Tensor, out: Optional[torch.Tensor] = None,
               k: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None, inverse: bool = False,
               stream=None) -> None:
        """x [rows, heads, head_dim] (bf16, fp16 or fp32, any row and head strides) rotated at
        ``positions`` [rows] into ``out`` (default: in place), and ``k`` likewise into ``k_out``.
        ``inverse``: the transposed map, the gradient of the call without it."""
        device, buf, dim = self.device, self._parts, rope.head_dim
        n, kind = x.shape[0], _TYPES.get(x.dtype)
        if kind is None:
            raise ValueError("x must be bfloat16, float16 or float32")
        self._here(positions)
        _int32_on_device("positions", positions, n)
        _put_heads(buf, 0, device, "x", x, x if out is None else out, dim)
        if k is not None:
            if k.dtype != x.dtype or k.shape[0] != n:
                raise ValueError("k must have x's type and rows")
            _put_heads(buf, _HEADS, device, "k", k, k if k_out is None else k_out, dim)
        status = self.lib.crf_rotary(self.h, rope.address, buf, 1 if k is None else 2, kind, n, positions.data_ptr(),
                                     inverse, _raw_stream(device) if stream is None else _stream(stream))
        if status:
            abi.check(status)

    def _pool_layer(self, pool: KVPool, layer: int) -> Tuple[int, int]:
        if not 0 <= layer < len(pool.k_pages):
            raise ValueError(f"layer {layer} is not in the pool")
        if pool.not_paged:
            raise ValueError(pool.not_paged)
        if pool.device != self.device:
            raise ValueError(f"the pool must be on cuda:{self.device}")
        return pool.n_kv_heads, pool.head_dim

    def _tables_here(self, device: int) -> None:
        if device != self.device:
            raise ValueError(f"the page tables must be on cuda:{self.device}")

    def cache_append(self, pool: KVPool, layer: int, chunks: Chunks, k: torch.Tensor, v: torch.Tensor,
                     q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                     rope: Optional[Rope] = None, stream=None) -> None:
        """Rows k, v [rows, kv heads, head_dim] into the requests' pages of ``layer``, k rotated at its
        position when ``rope`` is given; and ``q`` rotated into ``q_out`` (default: in place)."""
        hkv, dim = self._pool_layer(pool, layer)
        device, buf, n = self.device, self._parts, chunks.rows
        if chunks.device != device:
            raise ValueError(f"the page tables must be on cuda:{device}")
        if not chunks.append_ok:
            raise ValueError(f"page tables need {chunks.append_entries} entries to append")
        bf16 = torch.bfloat16
        if k.dtype != bf16 or v.dtype != bf16 or k.shape[0] != n or v.shape[0] != n or (
                q is not None and (q.dtype != bf16 or q.shape[0] != n)):
            raise ValueError(f"q, k and v must be bfloat16 with {n} rows")
        at = ctypes.addressof(buf)
        _put_heads(buf, _HEADS, device, "k", k, None, dim)
        _put_heads(buf, 2 * _HEADS, device, "v", v, None, dim)
        if q is not None:
            _put_heads(buf, 0, device, "q", q, q if q_out is None else q_out, dim)
        status = self.lib.crf_cache_append(self.h, None if rope is None else rope.address, pool.address, layer, hkv, dim,
                                           chunks.address, chunks.n, None if q is None else at, at + _HEADS,
                                           at + 2 * _HEADS, _raw_stream(device) if stream is None else _stream(stream))
        if status:
            abi.check(status)

    def chunk_attention_workspace(self, pool: KVPool, chunks: Chunks, n_q_heads: int, causal: bool = True,
                                  window: int = 0) -> torch.Tensor:
        """Workspace of a chunk_attention call; the same one serves every layer of the step."""
        hkv, dim = self._pool_layer(pool, 0)
        n = c_size_t()
        abi.check(self.lib.crf_chunk_attention_workspace_size(self.h, _fits("n_q_heads", n_q_heads), hkv, dim,
                                                              chunks.address, chunks.n, int(causal),
                                                              _fits("window", window), byref(n)))
        return torch.empty(max(256, n.value), dtype=torch.uint8, device=f"cuda:{self.device}")

    def chunk_attention(self, pool: KVPool, layer: int, chunks: Chunks, q: torch.Tensor, out: torch.Tensor,
                        workspace: torch.Tensor, lse: Optional[torch.Tensor] = None, scale: float = 0.0,
                        causal: bool = True, window: int = 0, stream=None) -> None:
        """out = attention of the rows q [rows, heads, head_dim] (bf16) over their requests' cached keys of
        ``layer`` (see crf_chunk_attention); ``lse`` fp32 [rows, heads]; ``scale`` 0: 1 / sqrt(head_dim)."""
        hkv, dim = self._pool_layer(pool, layer)
        device, buf, n = self.device, self._parts, chunks.rows
        if chunks.device != device:
            raise ValueError(f"the page tables must be on cuda:{device}")
        if not chunks.attend_ok:
            raise ValueError(f"page tables need {chunks.attend_entries} entries to attend")
        if q.dtype != torch.bfloat16 or q.shape[0] != n:
            raise ValueError(f"q must be bfloat16 with {n} rows")
        heads = _put_heads(buf, 0, device, "q", q, out, dim)
        self._here(workspace, lse)
        if lse is not None and (lse.dtype != torch.float32 or not lse.is_contiguous() or tuple(lse.shape) != (n, heads)):
            raise ValueError("lse must be a contiguous float32 [rows, heads]")
        if window:
            _fits("window", window)
        if 0 < scale < 2.0**-149:
            raise ValueError("scale would be 0 in float32, which stands for 1 / sqrt(head_dim)")
        status = self.lib.crf_chunk_attention(self.h, pool.address, layer, hkv, dim, chunks.address, chunks.n, buf,
                                              None if lse is None else lse.data_ptr(), scale, causal, window,
                                              workspace.data_ptr(), workspace.numel(),
                                              _raw_stream(device) if stream is None else _stream(stream))
        if status:
            abi.check(status)

    # -------------------------------------------------------------- pages
    def pages_workspace(self, num_pages: int, tables: PageTables) -> torch.Tensor:
        n = c_size_t()
        abi.check(self.lib.crf_pages_workspace_size(self.h, _fits("num_pages", num_pages), tables.address, tables.n, byref(n)))
        return torch.empty(max(256, n.value), dtype=torch.uint8, device=f"cuda:{self.device}")

    def _refs(self, num_pages: int, refs: torch.Tensor, refs_out: Optional[torch.Tensor]) -> Tuple[int, int]:
        self._here(refs, refs_out)
        out = refs if refs_out is None else refs_out
        for name, t in (("refs", refs), ("refs_out", out)):
            if t.numel() != num_pages:
                raise ValueError(f"{name} must have one count a page of the pool ({num_pages})")
            _int32_on_device(name, t, num_pages)
        return refs.data_ptr(), out.data_ptr()

    def pages_fork(self, pool: KVPool, refs: torch.Tensor, tables: PageTables, workspace: torch.Tensor,
                   refs_out: Optional[torch.Tensor] = None, deep: bool = False, stream=None) -> None:
        """A second continuation of every request into ``tables.outs``: whole pages shared, a part-filled
        last page (``deep``: every page) copied into the lowest free ones. ``refs`` is updated in place
        unless ``refs_out`` is given."""
        self._pages(self.lib.crf_pages_fork, pool, refs, refs_out, tables, workspace, stream, (int(deep),))

    def pages_compact(self, pool: KVPool, refs: torch.Tensor, tables: PageTables, workspace: torch.Tensor,
                      refs_out: Optional[torch.Tensor] = None, stream=None) -> None:
        """Live pages to the front of the pool; the tables with their new ids into ``tables.outs``."""
        self._pages(self.lib.crf_pages_compact, pool, refs, refs_out, tables, workspace, stream, ())

    def _pages(self, call, pool, refs, refs_out, tables, workspace, stream, flags) -> None:
        hkv, dim = self._pool_layer(pool, 0)
        if tables.outs is None:
            raise ValueError("the tables need outs")
        self._here(workspace)
        self._tables_here(tables.device)
        a, b = self._refs(pool.num_pages, refs, refs_out)
        status = call(self.h, pool.address, len(pool.k_pages), hkv, dim, a, b, tables.address, tables.n, *flags,
                      workspace.data_ptr(), workspace.numel(), self._stream_here(stream))
        if status:
            abi.check(status)

    def pages_release(self, refs: torch.Tensor, tables: PageTables, workspace: torch.Tensor,
                      refs_out: Optional[torch.Tensor] = None, stream=None) -> None:
        """Every table entry gives its reference back."""
        self._here(workspace)
        self._tables_here(tables.device)
        a, b = self._refs(refs.numel(), refs, refs_out)
        status = self.lib.crf_pages_release(self.h, refs.numel(), a, b, tables.address, tables.n, workspace.data_ptr(),
                                            workspace.numel(), self._stream_here(stream))
        if status:
            abi.check(status)

    def check(self, stream=None) -> None:
        abi.check(self.lib.crf_check(self.h, _stream(stream)))

    def selftest_timeout(self, stream=None) -> None:
        """Launch the bounded-wait self-test (its wait runs out after 2 s); the next check()
        raises CRF_ETIMEOUT."""
        abi.check(self.lib.crf_selftest_timeout(self.h, _stream(stream)))

    # -------------------------------------------------------------- profiling
    def profile_enable(self, on: bool = True, max_launches: int = 8192) -> None:
        abi.check(self.lib.crf_profile_enable(self.h, int(on), max_launches))

    def profile_read(self) -> Dict[str, Tuple[float, int]]:
        """{kernel kind: (total device ms, launches)} since the last read; also '_dropped'."""
        k = 32
        names = ctypes.create_string_buffer(k * 32)
        ms = (ctypes.c_double * k)()
        cnt = (ctypes.c_int * k)()
        n = ctypes.c_int()
        dropped = ctypes.c_int()
        abi.check(self.lib.crf_profile_read(self.h, k, names, ms, cnt, byref(n), byref(dropped)))
        out = {}
        for i in range(n.value):
            name = names.raw[i * 32:(i + 1) * 32].split(b"\0", 1)[0].decode()
            out[name] = (ms[i], cnt[i])
        out["_dropped"] = (0.0, dropped.value)
        return out


def kl_logits_noalloc(device: int, z_ref: torch.Tensor, z_cur: torch.Tensor, out_kl: torch.Tensor,
                      stream=None) -> None:
    """crf_kl_logits_noalloc: KL(softmax(z_ref) || softmax(z_cur)) per row with no workspace.

    For callers that cannot allocate device memory at call time; the library's fixed device
    scratch serves every call, so calls must not overlap on the GPU. The tensors are checked
    here (fp32, contiguous, same shape, on ``device``, out_kl long enough) because the library
    receives only their addresses.
    """
    if z_ref.dim() != 2 or tuple(z_cur.shape) != tuple(z_ref.shape):
        raise ValueError("z_ref and z_cur must be 2-D [n_rows, vocab] of the same shape")
    for name, t in (("z_ref", z_ref), ("z_cur", z_cur), ("out_kl", out_kl)):
        if t.dtype != torch.float32 or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous float32 tensor")
        if t.device.type != "cuda" or t.device.index != device:
            raise ValueError(f"{name} must be on cuda:{device}")
    if out_kl.numel() < z_ref.shape[0]:
        raise ValueError("out_kl holds fewer entries than z_ref has rows")
    if stream is None:
        stream = torch.cuda.current_stream(device)
    lib = abi.load()
    abi.check(lib.crf_kl_logits_noalloc(device, z_ref.data_ptr(), z_cur.data_ptr(),
                                        int(z_ref.shape[0]), int(z_ref.shape[1]),
                                        out_kl.data_ptr(), _stream(stream)))
