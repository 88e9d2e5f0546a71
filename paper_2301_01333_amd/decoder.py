"""A decoder's attention block over the entry points of include/ogc_decoder.h: head norms with rotary positions, the 4-bit cache, attention
over the prompt's own keys and, token by token, over the cache.

`python -m paper_2301_01333_amd.decoder` runs one on random projections: packed prompts of different lengths, then single tokens, and
prints what a call of each takes.  PyTorch owns memory and streams only.
"""
from __future__ import annotations

import argparse
from typing import Optional, Sequence

from . import binding


def check_rows(qkv, dtype, heads: int, head_dim: int, device) -> None:
    """ValueError unless qkv is rows as a layer's calls take them: the kernels get an address and strides, and believe them."""
    if qkv.dim() != 3 or tuple(qkv.shape[1:]) != (heads, head_dim):
        raise ValueError("rows of shape %s, not [tokens, %d, %d]" % (list(qkv.shape), heads, head_dim))
    if qkv.dtype != dtype:
        raise ValueError("rows of type %s, not %s" % (qkv.dtype, dtype))
    if qkv.stride(2) != 1:
        raise ValueError("the channels of a head are %d elements apart, not next to each other" % qkv.stride(2))
    if qkv.device != device:
        raise ValueError("rows on %s, not on %s" % (qkv.device, device))


def check_weights(q_weight, k_weight, dtype, head_dim: int) -> None:
    """ValueError unless there are weights of the type for queries and keys, or for neither."""
    if (q_weight is None) != (k_weight is None):
        raise ValueError("weights of the norms of queries and of keys, or neither")
    for w in (q_weight, k_weight):
        if w is not None and (w.dtype != dtype or tuple(w.shape) != (head_dim,) or not w.is_contiguous()):
            raise ValueError("a norm's weight of type %s and shape %s, not %s [%d], contiguous" % (w.dtype, list(w.shape), dtype, head_dim))


class DecoderAttention:
    """The attention of one layer for `batch` sequences of up to `max_tokens` tokens, whose keys and values are held in 4 bits.

    A call takes what the layer's projection leaves, rows [tokens][q_heads + 2 * kv_heads][head_dim], the sequences' new tokens one after
    the other, and returns the heads' outputs [tokens][q_heads][head_dim].  Calls are asynchronous on the current stream."""

    def __init__(self, dtype: str, q_heads: int, kv_heads: int, head_dim: int, batch: int, max_tokens: int, page_size: int = 64,
                 rot_dim: Optional[int] = None, layout: int = binding.OGC_ROPE_HALF, theta: float = 10000.0, q_weight=None, k_weight=None,
                 eps: float = 1e-6):
        import torch

        if dtype not in ("f32", "bf16"):
            raise ValueError("type %s, not f32 or bf16" % (dtype,))
        check_weights(q_weight, k_weight, torch.float32, head_dim)
        self.torch, self.dtype = torch, binding.DTYPES[dtype]
        self.torch_dtype = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
        self.q_heads, self.kv_heads, self.head_dim, self.batch, self.max_tokens = q_heads, kv_heads, head_dim, batch, max_tokens
        self.rot_dim, self.layout, self.eps = head_dim if rot_dim is None else rot_dim, layout, eps
        self.q_weight, self.k_weight = q_weight, k_weight
        if q_weight is not None and not (q_weight.is_cuda and k_weight.is_cuda):
            raise ValueError("the norms' weights are on %s and %s, not on the GPU" % (q_weight.device, k_weight.device))
        width = -(-max_tokens // page_size)
        self.cache_desc = binding.kv4_desc(kv_heads, head_dim, page_size, batch * width, batch, width)
        self.cache = torch.zeros(binding.ogc_kv4_cache_bytes(self.cache_desc), dtype=torch.uint8, device="cuda")
        self.table = torch.arange(batch * width, dtype=torch.int32, device="cuda").reshape(batch, width).contiguous()
        self.lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.held = 0  # tokens of the longest sequence, which launches are sized by
        half = torch.arange(0, self.rot_dim, 2, dtype=torch.float64, device="cuda")
        self.frequencies = theta ** (-half / max(self.rot_dim, 1))
        self.one_each = torch.arange(batch + 1, dtype=torch.int32, device="cuda")
        # for all steps, of any length: it never moves while a step or a captured graph may be using it
        each = (q_heads * head_dim, head_dim)
        longest = binding.kv4_attention_desc(self.dtype, q_heads, batch, 1, max_tokens, head_dim ** -0.5, each, each)
        need = binding.ogc_kv4_attention_workspace_bytes(self.cache_desc, longest)
        self.workspace = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")

    def _turned(self, qkv, positions):
        torch, n, hq, hk = self.torch, qkv.shape[0], self.q_heads, self.kv_heads
        q, k = qkv[:, :hq], qkv[:, hq:hq + hk]
        qo = torch.empty((n, hq, self.head_dim), dtype=self.torch_dtype, device="cuda")
        ko = torch.empty((n, hk, self.head_dim), dtype=self.torch_dtype, device="cuda")
        norm = int(self.q_weight is not None)
        desc = binding.rope_desc(self.dtype, n, hq, hk, self.head_dim, self.rot_dim, self.layout, norm, self.eps, 1.0, q.stride()[:2],
                                 k.stride()[:2], qo.stride()[:2], ko.stride()[:2])
        binding.ogc_rope_run(desc, q.data_ptr(), k.data_ptr(), self.q_weight.data_ptr() if norm else 0, self.k_weight.data_ptr() if norm else 0,
                             positions.data_ptr(), self.frequencies.data_ptr(), qo.data_ptr(), ko.data_ptr(), self._stream())
        return qo, ko, qkv[:, hq + hk:]

    def _stream(self) -> int:
        return int(self.torch.cuda.current_stream().cuda_stream)

    def _append(self, k, v, cu, longest):
        rows = binding.kv4_rows(self.dtype, k.shape[0], longest, k.stride()[:2], v.stride()[:2])
        binding.ogc_kv4_write(self.cache_desc, rows, k.data_ptr(), v.data_ptr(), cu.data_ptr(), self.lens.data_ptr(), self.table.data_ptr(),
                              self.cache.data_ptr(), self._stream())

    def prefill(self, qkv, lengths: Sequence[int]):
        """The prompts of empty sequences, packed; lengths: of all of them (zero: none)."""
        torch, hq, d = self.torch, self.q_heads, self.head_dim
        check_rows(qkv, self.torch_dtype, hq + 2 * self.kv_heads, d, self.cache.device)
        if len(lengths) != self.batch or sum(lengths) != qkv.shape[0] or min(lengths) < 0 or max(lengths) > self.max_tokens:
            raise ValueError("lengths %s do not fit %d sequences of up to %d tokens and %d rows" % (
                list(lengths), self.batch, self.max_tokens, qkv.shape[0]))
        ends = torch.tensor([0] + list(lengths), dtype=torch.int32).cumsum(0, dtype=torch.int32)
        cu = ends.cuda()
        positions = torch.cat([torch.arange(n, dtype=torch.int32) for n in lengths]).cuda()
        q, k, v = self._turned(qkv, positions)  # (a call that is refused leaves the layer as it is)
        self.lens.zero_()
        longest = max(lengths)
        self._append(k, v, cu, longest)
        o = torch.empty_like(q)
        desc = binding.prompt_desc(self.dtype, self.batch, hq, self.kv_heads, d, q.shape[0], k.shape[0], longest, longest, d ** -0.5, 1,
                                   q.stride()[:2], k.stride()[:2], v.stride()[:2], o.stride()[:2])
        binding.ogc_prompt_run(desc, q.data_ptr(), k.data_ptr(), v.data_ptr(), cu.data_ptr(), cu.data_ptr(), o.data_ptr(), self._stream())
        self.lens.copy_(ends[1:] - ends[:-1])
        self.held = longest
        return o

    def step(self, qkv):
        """One more token of every sequence, row b sequence b's."""
        torch = self.torch
        check_rows(qkv, self.torch_dtype, self.q_heads + 2 * self.kv_heads, self.head_dim, self.cache.device)
        if qkv.shape[0] != self.batch or self.held >= self.max_tokens:
            raise ValueError("%d rows for %d sequences, the longest of %d tokens of %d" % (qkv.shape[0], self.batch, self.held, self.max_tokens))
        q, k, v = self._turned(qkv, self.lens)
        self._append(k, v, self.one_each, 1)
        self.lens.add_(1)
        self.held += 1
        o = torch.empty_like(q)
        desc = binding.kv4_attention_desc(self.dtype, self.q_heads, self.batch, 1, self.held, self.head_dim ** -0.5, q.stride()[:2], o.stride()[:2])
        binding.ogc_kv4_attention_run(self.cache_desc, desc, q.data_ptr(), self.one_each.data_ptr(), self.lens.data_ptr(), self.table.data_ptr(),
                                      self.cache.data_ptr(), o.data_ptr(), self.workspace.data_ptr(), self._stream())
        return o


def main() -> None:
    ap = argparse.ArgumentParser(description="a decoder's attention block on random projections: prompts, then single tokens")
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="bf16")
    ap.add_argument("--heads", type=int, nargs=2, default=(32, 8), metavar=("QUERY", "KEY"))
    ap.add_argument("--head-dim", type=int, default=128)
    ap.add_argument("--prompts", type=int, nargs="+", default=[2048, 700, 1333, 96])
    ap.add_argument("--tokens", type=int, default=32, help="single tokens of every sequence after its prompt")
    a = ap.parse_args()
    import torch

    if not torch.cuda.is_available():
        raise SystemExit("no GPU")
    hq, hk = a.heads
    block = DecoderAttention(a.dtype, hq, hk, a.head_dim, len(a.prompts), max(a.prompts) + a.tokens,
                             q_weight=torch.ones(a.head_dim, device="cuda"), k_weight=torch.ones(a.head_dim, device="cuda"))
    make = lambda n: torch.randn((n, hq + 2 * hk, a.head_dim), device="cuda").to(block.torch_dtype)  # noqa: E731
    prompt, tokens = make(sum(a.prompts)), [make(len(a.prompts)) for _ in range(a.tokens)]
    marks = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
    block.prefill(prompt, a.prompts)  # (the first calls load the kernels)
    if a.tokens:
        block.step(tokens[0])
    marks[0].record()
    block.prefill(prompt, a.prompts)
    marks[1].record()
    for t in tokens:
        block.step(t)
    marks[2].record()
    torch.cuda.synchronize()
    print("prompts of %s tokens: %.1f us" % (a.prompts, marks[0].elapsed_time(marks[1]) * 1e3))
    if a.tokens:
        print("%d tokens of %d sequences: %.1f us each" % (a.tokens, len(a.prompts), marks[1].elapsed_time(marks[2]) * 1e3 / a.tokens))


if __name__ == "__main__":
    main()
