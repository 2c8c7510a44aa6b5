"""Device-memory plumbing around the binding: PyTorch allocates tensors and provides the stream;
every computation is a call into libslimattn."""
from __future__ import annotations

from dataclasses import dataclass
from typing import Optional, Sequence

import numpy as np
import torch

from . import binding as B


def bits_to_device(bits: np.ndarray, device="cuda:0") -> torch.Tensor:
    """uint16 bf16 bit patterns -> torch.bfloat16 tensor on the device."""
    return torch.from_numpy(bits.view(np.int16)).to(device).view(torch.bfloat16)


def device_to_f32(t: torch.Tensor) -> np.ndarray:
    """Device tensor (bf16 or f32) -> float32 numpy array (bf16 widened exactly)."""
    if t.dtype == torch.bfloat16:
        bits = t.view(torch.int16).cpu().numpy().view(np.uint16)
        return (bits.astype(np.uint32) << np.uint32(16)).view(np.float32)
    return t.cpu().numpy()


def f32_to_bf16_bits(x: np.ndarray) -> np.ndarray:
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    return ((u + np.uint32(0x7FFF) + ((u >> np.uint32(16)) & np.uint32(1))) >> np.uint32(16)).astype(np.uint16)


@dataclass
class Problem:
    """Device-resident inputs/outputs of one pack plus its tables."""
    tables: B.Tables
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    dtype: int
    scale: float
    q: torch.Tensor
    k: torch.Tensor
    v: torch.Tensor
    dO: torch.Tensor
    o: torch.Tensor
    lse: torch.Tensor
    dQ: torch.Tensor
    dK: torch.Tensor
    dV: torch.Tensor
    workspace: torch.Tensor

    def _kw(self, **over):
        kw = dict(n_q_heads=self.n_q_heads, n_kv_heads=self.n_kv_heads, head_dim=self.head_dim, dtype=self.dtype,
                  scale=self.scale, stream=torch.cuda.current_stream().cuda_stream)
        kw.update(over)
        return kw

    def forward(self, **over):
        B.fwd(self.q, self.k, self.v, self.tables, self.o, self.lse, **self._kw(**over))

    def backward(self, **over):
        B.bwd(self.q, self.k, self.v, self.o, self.lse, self.dO, self.tables, self.dQ, self.dK, self.dV,
              self.workspace, **self._kw(**over))

    def capture_step(self, flags: int = 0) -> "torch.cuda.CUDAGraph":
        """Forward + backward of the pack recorded into a HIP graph.  The two calls only launch kernels on the
        stream they are given (no allocation, no synchronisation, no memset), so a stream capture takes them as
        they are; per-kernel timing must be off (its events are not part of a capture).  Replaying the graph
        re-runs every launch on the same buffers."""
        g = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):                      # once outside the capture: first-call set-up is not recorded
            self.forward(flags=flags)
            self.backward(flags=flags)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=side):
            self.forward(flags=flags)
            self.backward(flags=flags)
        return g


def make_problem(q: np.ndarray, k: np.ndarray, v: np.ndarray, dO: np.ndarray, cu, slices, fwd_units, bwd_units, *,
                 bf16: bool, scale: Optional[float] = None, device="cuda:0") -> Problem:
    """Uploads float32 host arrays (bf16-exact when bf16=True) and allocates outputs + workspace."""
    T, hq, d = q.shape
    hkv = k.shape[1]
    torch.cuda.set_device(device)
    tables = B.tables_create(cu, slices, fwd_units[0], fwd_units[1], bwd_units[0], bwd_units[1])
    if bf16:
        up = lambda a: bits_to_device(f32_to_bf16_bits(a), device)
        tdt = torch.bfloat16
    else:
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(device)
        tdt = torch.float32
    dq_, dk_, dv_, do_ = up(q), up(k), up(v), up(dO)
    ws = torch.empty(max(B.bwd_workspace_bytes(tables, hq, hkv, d), 256), dtype=torch.uint8, device=device)
    return Problem(tables, hq, hkv, d, B.BF16 if bf16 else B.F32, float(scale if scale is not None else d ** -0.5),
                   dq_, dk_, dv_, do_,
                   torch.empty((T, hq, d), dtype=tdt, device=device), torch.empty((hq, T), dtype=torch.float32, device=device),
                   torch.empty((T, hq, d), dtype=tdt, device=device), torch.empty((T, hkv, d), dtype=tdt, device=device),
                   torch.empty((T, hkv, d), dtype=tdt, device=device), ws)


def _here():
    """Index of the current GPU and handle of its current stream, without the object around it (3 us of a call that took 11)."""
    if not torch.cuda.is_initialized():
        torch.cuda.init()
    dev = torch._C._cuda_getDevice()
    return dev, torch._C._cuda_getCurrentRawStream(dev)


def _lib_dtype(dtype: torch.dtype) -> int:
    if dtype == torch.bfloat16:
        return B.BF16
    if dtype == torch.float32:
        return B.F32
    raise ValueError(f"{dtype}: expected torch.bfloat16 or torch.float32")


class Rotary:
    """Norm per head and rotation of a layer's queries and keys, in front of slimattn_fwd, and their gradients behind slimattn_bwd: the
    parameters of the layer and what its backward pass needs (workspace, weight gradients), for calls of any number of tokens.
    One backward call at a time where it has a norm (its workspace, `dq_weight`, `dk_weight`)."""

    def __init__(self, n_q_heads: int, n_kv_heads: int, head_dim: int, dtype: torch.dtype, inv_freq: Optional[torch.Tensor], *,
                 q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None, norm: bool = False, eps: float = 1e-6,
                 rotary_dim: Optional[int] = None, sections: Optional[Sequence[int]] = None, dealt: bool = False, adjacent: bool = False,
                 device="cuda"):
        if not norm and (q_weight is not None or k_weight is not None):
            raise ValueError("q_weight, k_weight: weights of the norm, given without norm=True")
        self.n_q_heads, self.n_kv_heads, self.head_dim = n_q_heads, n_kv_heads, head_dim
        self.inv_freq, self.q_weight, self.k_weight, self.norm = inv_freq, q_weight, k_weight, norm
        rotary_dim = head_dim if rotary_dim is None else rotary_dim
        self._shape = (n_q_heads, n_kv_heads, head_dim, _lib_dtype(dtype), rotary_dim, tuple(sections) if sections is not None else (rotary_dim // 2,),
                       eps, B.ROPE_NORM * norm | B.ROPE_ADJACENT * adjacent | B.ROPE_DEALT * dealt)
        self.dq_weight = self.dk_weight = self.workspace = None
        if norm:
            need = B.rope_bwd_workspace_bytes(0, *self._shape)
            self.workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=device)
            self.dq_weight = torch.zeros(head_dim, dtype=torch.float32, device=device)
            self.dk_weight = torch.zeros(head_dim, dtype=torch.float32, device=device)

    def forward(self, q, k, positions, q_out, k_out):
        """q, k [T, heads, d] (columns of a fused projection, or packed), positions int32 [axes, T] or [T] -> q_out, k_out, packed."""
        B._rope_fwd(*_here(), (q if q is not None else k).shape[0], self._shape, q, k, positions, self.inv_freq, self.q_weight, self.k_weight, q_out, k_out)

    def backward(self, q, k, positions, dq_out, dk_out, dq, dk):
        """dQ, dK of the attention and the forward's inputs -> dq, dk; the weights' gradients go to dq_weight, dk_weight."""
        B._rope_bwd(*_here(), (dq_out if dq_out is not None else dk_out).shape[0], self._shape, q, k, positions, self.inv_freq, self.q_weight,
                    self.k_weight, dq_out, dk_out, dq, dk, self.dq_weight, self.dk_weight, self.workspace)


class KVCache:
    """One layer's keys and values of a batch of sequences in 4 bits: the pages, the page table and the lengths (device tensors the program
    updates as sequences grow), and the workspace of attention calls of up to `max_rows` rows (and of one row a sequence).  One attention
    call at a time: two streams, or two recorded graphs that may run together, need a handle each (`cache` may be shared)."""

    def __init__(self, n_pages: int, page_size: int, n_kv_heads: int, head_dim: int, dtype: torch.dtype, page_table: torch.Tensor,
                 lens: torch.Tensor, *, max_rows: int = 0, n_q_heads: int = 0):
        self.page_table, self.lens, self.n_q_heads = page_table, lens, n_q_heads
        self._shape = dict(n_pages=n_pages, page_size=page_size, n_kv_heads=n_kv_heads, head_dim=head_dim, dtype=_lib_dtype(dtype),
                           n_seqs=page_table.shape[0], max_pages=page_table.shape[1])
        self._values = tuple(self._shape.values())
        size = B.cache_bytes(n_pages, page_size, n_kv_heads, head_dim)
        if size == 0:
            raise ValueError("cache: unsupported pages or heads")
        self.cache = torch.empty(size, dtype=torch.uint8, device=page_table.device)
        self.workspace = None
        if n_q_heads:
            need = B.cache_attn_workspace_bytes(n_q_heads, n_rows=max(max_rows, page_table.shape[0]), **self._shape)
            self.workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=page_table.device)

    def write(self, k, v, row_ptr=None):
        """k, v [rows, Hkv, d]: the last tokens of the sequences (row_ptr: first row of each; None: one each) into their pages."""
        B._cache_write(*_here(), k.shape[0], self._values, k, v, self.cache, self.page_table, self.lens, row_ptr)

    def read(self, k, v, row_ptr=None):
        """The last tokens of the sequences from their pages -> k, v."""
        B._cache_read(*_here(), k.shape[0], self._values, self.cache, self.page_table, self.lens, row_ptr, k, v)

    def attend(self, q, o, lse, scale, row_ptr=None):
        """q [rows, Hq, d], the queries of the sequences' last tokens, over their pages -> o, lse [Hq, rows] (or None)."""
        B._cache_attn(*_here(), q.shape[0], self._values, self.n_q_heads, scale, q, self.cache, self.page_table, self.lens, row_ptr, o, lse, self.workspace)
