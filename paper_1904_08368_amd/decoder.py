"""An attention layer that is served from a paged cache, as a sequence of fused primitive functions on preallocated buffers (paper Section 3.3).

One layer is four calls of the library, for a prompt's many tokens as for one new token of each sequence:
  relay_qdense_w4 (queries, keys, values)  ->  relay_rope_append  ->  relay_paged_attention  ->  relay_qdense_w4 with the residual.
Packing of the weights, the table of angles and the buffers are compile-time work and happen in the constructors; a call of a layer only
enqueues kernels on torch's current stream, so it can be captured into a HIP graph and replayed while the sequences grow.

    cache = PagedCache(layers, pages=4096, page_size=16, kv_heads=8, head_dim=128)
    ids = [cache.open() for _ in prompts]
    step = Step(cache, batch=len(ids), tokens=sum(map(len, prompts)), max_q_len=max(map(len, prompts)), max_kv_len=8192)
    step.extend(ids, [len(p) for p in prompts])          # slots for the new tokens; what the kernels read goes to the device
    for i, layer in enumerate(layers):
        x = layer(x, i, step)
"""
from __future__ import annotations

import math
from typing import Dict, List, Optional, Sequence

import numpy as np
import torch

from . import binding as B


class PagedCache:
    """Keys and values of all layers in pages of `page_size` slots, dealt out to sequences as these grow.  A page number means the same page
    in every layer."""

    def __init__(self, layers: int, pages: int, page_size: int, kv_heads: int, head_dim: int, dtype=torch.float16, device: str = "cuda:0"):
        shape = (layers, pages, page_size, kv_heads, head_dim)
        self.k, self.v = torch.zeros(shape, dtype=dtype, device=device), torch.zeros(shape, dtype=dtype, device=device)
        self.page_size = page_size
        self.free: List[int] = list(range(pages - 1, -1, -1))
        self.pages: Dict[int, List[int]] = {}
        self.length: Dict[int, int] = {}
        self._next = 0

    def open(self) -> int:
        """A new sequence without tokens."""
        self._next += 1
        self.pages[self._next], self.length[self._next] = [], 0
        return self._next

    def close(self, seq: int) -> None:
        """The sequence's pages are free again."""
        self.free.extend(reversed(self.pages.pop(seq)))
        del self.length[seq]

    def extend(self, seqs: Sequence[int], new: Sequence[int]) -> None:
        """Room for `new` more tokens of each sequence; all of it or, if the pages do not suffice, none."""
        if len(set(seqs)) != len(seqs) or len(new) != len(seqs) or min(new, default=0) < 0:
            raise ValueError("each sequence once, with its number of new tokens")
        need = [-(-(self.length[s] + n) // self.page_size) - len(self.pages[s]) for s, n in zip(seqs, new)]
        if sum(need) > len(self.free):
            raise MemoryError(f"{sum(need)} pages needed, {len(self.free)} free")
        for s, n, p in zip(seqs, new, need):
            self.pages[s].extend(self.free.pop() for _ in range(p))
            self.length[s] += n


class Step:
    """What the kernels of one step read about its tokens, in device tensors of fixed extents: batch, tokens, and the longest of both that
    a sequence may reach.  extend() refills them, so a captured step can be replayed for the next tokens."""

    def __init__(self, cache: PagedCache, batch: int, tokens: int, max_q_len: int, max_kv_len: int):
        self.cache, self.max_q_len, self.max_kv_len = cache, max_q_len, max_kv_len
        self.batch, self.tokens = batch, tokens
        self.per_seq = -(-max_kv_len // cache.page_size)
        device = cache.k.device

        def ints(*shape, value=0):
            return torch.full(shape, value, dtype=torch.int32, device=device)

        # (no tokens yet: run before the first extend(), say to warm up before a capture, a step stores nothing)
        self.page_table, self.q_starts, self.kv_lens = ints(batch, self.per_seq, value=-1), ints(batch + 1), ints(batch)
        self.positions, self.slots = ints(tokens), ints(tokens, value=-1)

    def extend(self, seqs: Sequence[int], new: Sequence[int]) -> None:
        """new[b] more tokens of sequence seqs[b], in this order in the rows of the layers' input; rows behind the last are padding."""
        if len(set(seqs)) != len(seqs) or len(seqs) > self.batch or len(new) != len(seqs) or min(new, default=0) < 0 or \
                sum(new) > self.tokens or max(new, default=0) > self.max_q_len:
            raise ValueError("the sequences and their new tokens do not fit this step")
        before = [self.cache.length[s] for s in seqs]
        if any(k + n > self.max_kv_len for k, n in zip(before, new)):
            raise ValueError(f"a sequence would pass {self.max_kv_len} tokens")
        self.cache.extend(seqs, new)
        table, starts = np.full((self.batch, self.per_seq), -1, np.int32), np.zeros(self.batch + 1, np.int32)
        lens, positions, slots = np.zeros(self.batch, np.int32), np.zeros(self.tokens, np.int32), np.full(self.tokens, -1, np.int32)
        at = 0
        for b, (s, k, n) in enumerate(zip(seqs, before, new)):
            pages = np.array(self.cache.pages[s], np.int32)
            table[b, :len(pages)] = pages
            p = np.arange(k, k + n, dtype=np.int32)
            positions[at:at + n] = p
            slots[at:at + n] = pages[p // self.cache.page_size] * self.cache.page_size + p % self.cache.page_size
            lens[b], at = k + n, at + n
            starts[b + 1] = at
        starts[len(seqs) + 1:] = at
        for dst, src in ((self.page_table, table), (self.q_starts, starts), (self.kv_lens, lens), (self.positions, positions), (self.slots, slots)):
            dst.copy_(torch.from_numpy(src))


class Dense4:
    """A dense layer with 4-bit weights, packed for the kernels: codes uint8 [n, k/2], scales [n, groups], zero points uint8 or None."""

    def __init__(self, codes, scales, zeros, group: int, k: int, bias: Optional[torch.Tensor] = None):
        self.n, self.k, self.group, self.zeros, self.bias, self.dtype = codes.shape[0], k, group, zeros, bias, scales.dtype
        x, y = (torch.empty((0, e), dtype=self.dtype, device=codes.device) for e in (k, self.n))
        d = B.qdense_w4_desc(x, y, group, zeros, bias)
        self.packed = torch.empty(B.relay_qdense_w4_packed_bytes(d), dtype=torch.uint8, device=codes.device)
        B.relay_prepack_qdense_w4(d, codes, scales, zeros, self.packed)

    def __call__(self, x, y, residual=None):
        # (the packed order depends on all of these, and nothing of it is left in the packed bytes)
        if x.dtype != self.dtype or x.shape[1] != self.k or y.shape[1] != self.n:
            raise ValueError(f"x {tuple(x.shape)} of {x.dtype} and y {tuple(y.shape)} do not go with a layer of {self.n} units by {self.k} in {self.dtype}")
        d = B.qdense_w4_desc(x, y, self.group, self.zeros, self.bias, residual)
        d.packed_bytes = self.packed.nbytes   # (known here: not asked for again)
        B.relay_qdense_w4(d, x, self.packed, self.bias, residual, y)
        return y


def quantize4(w: torch.Tensor, group: int):
    """codes, scales and zero points of a weight matrix [n, k], each group of a row between its least and its largest value.

    The least scale: fp16's 2^-20, which it still holds to 5 bits (its least normal number, 2^-14, would take all of a group's codes from
    weights below 2^-15), bf16's least normal number."""
    n, k = w.shape
    groups = -(-k // group)
    parts = torch.nn.functional.pad(w.float(), (0, groups * group - k), value=0.0).view(n, groups, group)
    lo, hi = parts.amin(2).clamp(max=0.0), parts.amax(2).clamp(min=0.0)
    scales = ((hi - lo) / 15).clamp(min=2.0 ** -20 if w.dtype == torch.float16 else torch.finfo(w.dtype).tiny).to(w.dtype)
    zeros = (-lo / scales.float()).round().clamp(0, 15)
    codes = (parts / scales.float()[..., None] + zeros[..., None]).round().clamp(0, 15).to(torch.uint8).view(n, -1)[:, :k]
    return (codes[:, 0::2] | codes[:, 1::2] << 4).contiguous(), scales.contiguous(), zeros.to(torch.uint8).contiguous()


class Workspace:
    """Scratch that grows to the largest call; for calls that follow each other on one stream.

    A captured step holds the address of the buffer it was captured with, so a buffer that a larger one has replaced stays alive as long as the
    workspace (each is at least twice as large as the one before: together they are below two of the last).  A call that needs more while
    a graph is captured gets scratch of the graph's own, cleared on every replay: the fill that clears a buffer is only recorded then, and calls outside
    of the graph would find whatever the memory held before.  Run a step once before it is captured, and it needs none."""

    def __init__(self):
        self.buffer: Optional[torch.Tensor] = None
        self._outgrown: List[torch.Tensor] = []

    def of(self, nbytes: int, device) -> Optional[torch.Tensor]:
        if not nbytes or (self.buffer is not None and self.buffer.numel() >= nbytes):
            return self.buffer
        if torch.cuda.is_available() and torch.cuda.is_current_stream_capturing():
            return torch.zeros(nbytes, dtype=torch.uint8, device=device)
        if self.buffer is not None:
            self._outgrown.append(self.buffer)
            nbytes = max(nbytes, 2 * self.buffer.numel())
        self.buffer = torch.zeros(nbytes, dtype=torch.uint8, device=device)
        return self.buffer


class AttentionLayer:
    """x + W_o attention(W_qkv x) over the cache.  qkv: Dense4 of (q_heads + 2 kv_heads) * head_dim units, out: Dense4 back to x's width;
    cos_sin: the table of relay_rope_table.  One workspace serves the layers of a stack: pass the first one's."""

    def __init__(self, qkv: Dense4, out: Dense4, cos_sin, q_heads: int, kv_heads: int, head_dim: int, max_tokens: int, style=B.ROPE_HALF,
                 window: int = 0, scale: Optional[float] = None, workspace: Optional[Workspace] = None):
        if qkv.n != (q_heads + 2 * kv_heads) * head_dim or out.k != q_heads * head_dim or out.n != qkv.k:
            raise ValueError("the projections and the heads do not go together")
        self.qkv, self.out, self.cos_sin, self.style, self.window = qkv, out, cos_sin, style, window
        self.heads, self.scale = (q_heads, kv_heads, head_dim), 1 / math.sqrt(head_dim) if scale is None else scale
        self.workspace = Workspace() if workspace is None else workspace
        device = qkv.packed.device
        self._qkv = torch.empty((max_tokens, qkv.n), dtype=qkv.dtype, device=device)
        # (rows of padding are read by the second projection and written by nothing: what the memory held before would be their input)
        self._attn = torch.zeros((max_tokens, q_heads * head_dim), dtype=qkv.dtype, device=device)

    def __call__(self, x, index: int, step: Step, y=None):
        """x [step.tokens, width] -> y; `index`: this layer's cache."""
        q_heads, kv_heads, dim = self.heads
        y = torch.empty_like(x) if y is None else y
        kc, vc = step.cache.k[index], step.cache.v[index]
        qkv, attn = self._qkv[:step.tokens], self._attn[:step.tokens].view(step.tokens, q_heads, dim)
        self.qkv(x, qkv)
        q, k, v = (t.unflatten(1, (-1, dim)) for t in qkv.split((q_heads * dim, kv_heads * dim, kv_heads * dim), dim=1))
        B.relay_rope_append(B.rope_append_desc(q, k, v, self.cos_sin, q, kc, self.style), q, k, v, self.cos_sin, step.positions, step.slots, q, kc, vc)
        d = B.paged_attention_desc(q, kc, step.page_table, attn, step.max_q_len, step.max_kv_len, self.scale, True, self.window)
        ws = self.workspace.of(B.relay_paged_attention_workspace_bytes(d), x.device)
        B.relay_paged_attention(d, q, kc, vc, step.page_table, step.q_starts, step.kv_lens, attn, ws)
        return self.out(attn.flatten(1), y, residual=x)
