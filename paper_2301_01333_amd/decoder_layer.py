"""A decoder's layer over the entry points of include/ogc_mx.h and its attention block (decoder.py), and the choice of the next tokens (include/ogc_sample.h):
weights in 4 bits, the rows between them in 8 or 4.

`python -m paper_2301_01333_amd.decoder_layer` runs layers with random weights: packed prompts of different lengths, then single tokens, each of them
chosen from the logits of the one before, and prints what a call of each takes.  PyTorch owns memory and streams only.
"""
from __future__ import annotations

import argparse
from typing import Optional, Sequence

from . import binding
from .decoder import DecoderAttention

FORMATS = {"mx4": binding.OGC_MX4, "mx8": binding.OGC_MX8}
NORMS = {"same": binding.OGC_NORM_SAME, "mx4": binding.OGC_NORM_MX4, "mx8": binding.OGC_NORM_MX8}


def _types():
    import torch

    return {torch.float32: binding.OGC_F32, torch.bfloat16: binding.OGC_BF16}


def _type(dtype, what: str) -> int:
    if dtype not in _types():
        raise ValueError("%s of %s, not float32 or bfloat16" % (what, dtype))
    return _types()[dtype]


def _stream() -> int:
    import torch

    return int(torch.cuda.current_stream().cuda_stream)


def on_this_gpu(x) -> bool:
    import torch

    return x.is_cuda and x.device.index == torch.cuda.current_device()


def check_matrix(x, what: str, channels: Optional[int] = None) -> None:
    """ValueError unless x is rows as the calls take them: the kernels get an address and a stride, and believe them."""
    if x.dim() != 2 or (channels is not None and x.shape[1] != channels):
        raise ValueError("%s of shape %s, not [rows, %s]" % (what, list(x.shape), "channels" if channels is None else channels))
    _type(x.dtype, what)
    if x.shape[1] > 1 and x.stride(1) != 1:
        raise ValueError("the channels of %s are %d elements apart, not next to each other" % (what, x.stride(1)))
    if x.shape[0] > 1 and (x.stride(0) < x.shape[1] or x.stride(0) * x.element_size() % 16):
        raise ValueError("the rows of %s are %d elements apart, not a multiple of 16 bytes from %d on" % (what, x.stride(0), x.shape[1]))
    if not on_this_gpu(x) or x.data_ptr() % 16:
        raise ValueError("%s on %s at %d, not on the current GPU at a multiple of 16 bytes" % (what, x.device, x.data_ptr()))


def _stride(x) -> int:
    return x.stride(0) if x.shape[0] > 1 else -(-x.shape[1] // 8) * 8  # (of a single row it says nothing)


def _rows(n: int, c: int, dtype):
    """Rows to be written: [n, c], a multiple of 16 bytes apart."""
    import torch

    return torch.empty((n, -(-c // 8) * 8), dtype=dtype, device="cuda")[:, :c]


class MxMatrix:
    """A microscaled matrix on the GPU: rows of 32-channel groups with a power of two each, in the matrix instruction's order."""

    def __init__(self, fmt: str, rows: int, channels: int):
        import torch

        if fmt not in FORMATS:
            raise ValueError("format %s, not mx4 or mx8" % (fmt,))
        self.fmt, self.rows, self.channels = fmt, rows, channels
        codes, scales = binding.ogc_mx_bytes(FORMATS[fmt], rows, channels)
        self.codes, self.scales = (torch.empty(max(n, 16), dtype=torch.uint8, device="cuda") for n in (codes, scales))

    @classmethod
    def write(cls, x, fmt: str, gate: bool = False) -> "MxMatrix":
        """The rows of x; gate: x has a gate and then a value for each channel, and silu(gate) * value is written."""
        check_matrix(x, "rows")
        if gate and x.shape[1] % 2:
            raise ValueError("%d channels are no pairs of a gate and a value" % x.shape[1])
        m = cls(fmt, x.shape[0], x.shape[1] // 2 if gate else x.shape[1])
        rows = binding.mx_rows(_types()[x.dtype], FORMATS[fmt], m.rows, m.channels, int(gate), _stride(x))
        binding.ogc_mx_write(rows, x.data_ptr(), m.codes.data_ptr(), m.scales.data_ptr(), _stream())
        return m

    def check(self, what: str) -> None:
        """ValueError unless the matrix is on the current GPU."""
        if not on_this_gpu(self.codes):
            raise ValueError("%s on %s, not on the current GPU" % (what, self.codes.device))

    def read(self, dtype):
        kind = _type(dtype, "rows")
        self.check("a matrix")
        y = _rows(self.rows, self.channels, dtype)
        rows = binding.mx_rows(kind, FORMATS[self.fmt], self.rows, self.channels, 0, _stride(y))
        binding.ogc_mx_read(rows, self.codes.data_ptr(), self.scales.data_ptr(), y.data_ptr(), _stream())
        return y


def add_norm(x, residual, weight, eps: float = 1e-6, out: str = "same"):
    """(x + residual, its root-mean-square norm as rows or as a matrix); without a residual (None): (x, its norm)."""
    import torch

    if out not in NORMS:
        raise ValueError("a norm as %s, not same, mx4 or mx8" % (out,))
    check_matrix(x, "rows")
    if residual is not None:
        check_matrix(residual, "the residual", x.shape[1])
        if residual.shape[0] != x.shape[0] or residual.dtype != x.dtype or residual.device != x.device:
            raise ValueError("a residual of %d rows of %s on %s for %d of %s on %s" % (residual.shape[0], residual.dtype, residual.device, x.shape[0], x.dtype, x.device))
    if weight.dtype != torch.float32 or tuple(weight.shape) != (x.shape[1],) or not weight.is_contiguous() or weight.device != x.device or weight.data_ptr() % 16:
        raise ValueError("a weight of %s %s on %s, not float32 [%d], contiguous, on %s" % (weight.dtype, list(weight.shape), weight.device, x.shape[1], x.device))
    n, c = x.shape
    s = x if residual is None else _rows(n, c, x.dtype)
    y = _rows(n, c, x.dtype) if out == "same" else MxMatrix(out, n, c)
    desc = binding.norm_desc(_types()[x.dtype], n, c, NORMS[out], eps, _stride(x), 0 if residual is None else _stride(residual),
                             0 if residual is None else _stride(s), _stride(y) if out == "same" else 0)
    binding.ogc_norm_run(desc, x.data_ptr(), 0 if residual is None else residual.data_ptr(), weight.data_ptr(), 0 if residual is None else s.data_ptr(),
                         y.data_ptr() if out == "same" else y.codes.data_ptr(), 0 if out == "same" else y.scales.data_ptr(), _stream())
    return s, y


class Projection:
    """y = x w^T + bias with weights [n, k] held in 4 bits."""

    def __init__(self, weight, bias=None):
        import torch

        self.weight = MxMatrix.write(weight, "mx4")
        if bias is not None and (bias.dtype != torch.float32 or tuple(bias.shape) != (weight.shape[0],) or not bias.is_contiguous() or bias.device != weight.device):
            raise ValueError("a bias of %s %s, not float32 [%d], contiguous, on %s" % (bias.dtype, list(bias.shape), weight.shape[0], weight.device))
        self.bias = bias

    def __call__(self, x: MxMatrix, dtype):
        if x.channels != self.weight.channels:
            raise ValueError("rows of %d channels for weights of %d" % (x.channels, self.weight.channels))
        kind = _type(dtype, "a result")
        x.check("rows")
        self.weight.check("weights")
        n = self.weight.rows
        y = _rows(x.rows, n, dtype)
        desc = binding.mx_product_desc(kind, FORMATS[x.fmt], binding.OGC_MX4, x.rows, n, x.channels, int(self.bias is not None), _stride(y))
        binding.ogc_mx_product_run(desc, x.codes.data_ptr(), x.scales.data_ptr(), self.weight.codes.data_ptr(), self.weight.scales.data_ptr(),
                                   self.bias.data_ptr() if self.bias is not None else 0, y.data_ptr(), 0, _stream())
        return y


class DecoderLayer:
    """Norm, attention, norm, gated feed-forward.  A call takes the residual's rows [tokens, channels] and what the layer before adds to them (None:
    nothing), and returns the same for the next layer: each sum meets its norm in one pass.

    attention: a DecoderAttention of the layer's heads.  Weights: qkv [heads * head_dim, channels] of queries, keys and values, out [channels, query heads *
    head_dim], gate_up [2 * hidden, channels], down [channels, hidden]; norms fp32 [channels].  rows: the format of the rows between them.  A layer's calls belong on one stream, one after
    the other, or in graphs that are replayed so: they share the attention's cache and its workspace."""

    def __init__(self, attention: DecoderAttention, qkv, out, gate_up, down, norm_attention, norm_feed_forward, eps: float = 1e-6, rows: str = "mx8"):
        a, c = attention, out.shape[0]
        heads, hidden = a.q_heads + 2 * a.kv_heads, down.shape[1]
        for w, want, what in ((qkv, (heads * a.head_dim, c), "qkv"), (out, (c, a.q_heads * a.head_dim), "out"), (gate_up, (2 * hidden, c), "gate_up"), (down, (c, hidden), "down")):
            if tuple(w.shape) != want:
                raise ValueError("%s weights of shape %s, not %s" % (what, list(w.shape), list(want)))
        if rows not in FORMATS:
            raise ValueError("format %s, not mx4 or mx8" % (rows,))
        self.attention, self.channels, self.eps, self.rows = a, c, eps, rows
        self.qkv, self.out, self.gate_up, self.down = (Projection(w) for w in (qkv, out, gate_up, down))
        self.norm_attention, self.norm_feed_forward = norm_attention, norm_feed_forward

    def _layer(self, x, more, attend):
        a, dtype = self.attention, self.attention.torch_dtype
        check_matrix(x, "rows", self.channels)
        if x.dtype != dtype:
            raise ValueError("rows of %s, not %s" % (x.dtype, dtype))
        x, normed = add_norm(x, more, self.norm_attention, self.eps, self.rows)
        o = attend(self.qkv(normed, dtype).unflatten(1, (-1, a.head_dim)))
        more = self.out(MxMatrix.write(o.flatten(1), self.rows), dtype)
        x, normed = add_norm(more, x, self.norm_feed_forward, self.eps, self.rows)
        return x, self.down(MxMatrix.write(self.gate_up(normed, dtype), self.rows, gate=True), dtype)

    def prefill(self, x, more, lengths: Sequence[int]):
        """The prompts of empty sequences, packed, as DecoderAttention.prefill takes them."""
        return self._layer(x, more, lambda qkv: self.attention.prefill(qkv, lengths))

    def step(self, x, more):
        """One more token of every sequence."""
        return self._layer(x, more, self.attention.step)


class TokenChoice:
    """Chooses a token of each of `rows` rows of `vocab` logits: temperature, top-k, top-p and min-p as tensors [rows] (None: 1, and no limit).
    Every call has a workspace of its own, from PyTorch's pool of its stream or graph, so that calls on several streams, and captured ones, may run at the same time."""

    def __init__(self, rows: int, vocab: int, dtype, temperature=None, top_k=None, top_p=None, min_p=None):
        import torch

        _type(dtype, "logits")
        for t, kind, what in ((temperature, torch.float32, "temperature"), (top_k, torch.int32, "top_k"), (top_p, torch.float32, "top_p"), (min_p, torch.float32, "min_p")):
            if t is not None and (t.dtype != kind or tuple(t.shape) != (rows,) or not t.is_contiguous() or not on_this_gpu(t)):
                raise ValueError("%s of %s %s on %s, not %s [%d], contiguous, on the GPU" % (what, t.dtype, list(t.shape), t.device, kind, rows))
        self.rows, self.vocab, self.dtype, self.limits = rows, vocab, dtype, (temperature, top_k, top_p, min_p)
        self.device = torch.device("cuda", torch.cuda.current_device())
        # (for rows of any stride)
        self.workspace_bytes = max(16, binding.ogc_sample_workspace_bytes(binding.sample_desc(_types()[dtype], rows, vocab, vocab)))

    def __call__(self, logits, uniform):
        """(tokens int32 [rows], their log-probabilities float32 [rows]); uniform: float32 [rows], random numbers from 0 to 1."""
        import torch

        if tuple(logits.shape) != (self.rows, self.vocab) or logits.dtype != self.dtype or not on_this_gpu(logits) or (self.vocab > 1 and logits.stride(1) != 1):
            raise ValueError("logits of %s %s on %s, not %s [%d, %d], next to each other, on the GPU" % (logits.dtype, list(logits.shape), logits.device, self.dtype, self.rows, self.vocab))
        if self.device != logits.device:
            raise ValueError("logits on %s, the limits on %s" % (logits.device, self.device))
        if uniform.dtype != torch.float32 or tuple(uniform.shape) != (self.rows,) or not uniform.is_contiguous() or uniform.device != logits.device:
            raise ValueError("uniform of %s %s on %s, not float32 [%d], contiguous, on %s" % (uniform.dtype, list(uniform.shape), uniform.device, self.rows, logits.device))
        tokens = torch.empty(self.rows, dtype=torch.int32, device="cuda")
        logs = torch.empty(self.rows, dtype=torch.float32, device="cuda")
        space = torch.empty(self.workspace_bytes, dtype=torch.uint8, device="cuda")
        desc = binding.sample_desc(_types()[self.dtype], self.rows, self.vocab, logits.stride(0) if self.rows > 1 else self.vocab)
        binding.ogc_sample_run(desc, logits.data_ptr(), *(0 if t is None else t.data_ptr() for t in self.limits), uniform.data_ptr(), tokens.data_ptr(), logs.data_ptr(),
                               space.data_ptr(), _stream())
        return tokens, logs


def main() -> None:
    ap = argparse.ArgumentParser(description="a decoder's layers with random weights: prompts, then single tokens chosen from the logits")
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="bf16")
    ap.add_argument("--rows", choices=sorted(FORMATS), default="mx8", help="format of the rows between projections")
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--channels", type=int, default=4096)
    ap.add_argument("--hidden", type=int, default=12288)
    ap.add_argument("--heads", type=int, nargs=2, default=(32, 8), metavar=("QUERY", "KEY"))
    ap.add_argument("--head-dim", type=int, default=128)
    ap.add_argument("--vocab", type=int, default=32000)
    ap.add_argument("--prompts", type=int, nargs="+", default=[512, 700, 333, 96])
    ap.add_argument("--tokens", type=int, default=32, help="single tokens of every sequence after its prompt")
    a = ap.parse_args()
    import torch

    if not torch.cuda.is_available():
        raise SystemExit("no GPU")
    (hq, hk), d, c, batch = a.heads, a.head_dim, a.channels, len(a.prompts)
    dtype = {"f32": torch.float32, "bf16": torch.bfloat16}[a.dtype]
    random = lambda n, k: torch.randn((n, k), device="cuda") * k ** -0.5  # noqa: E731
    ones = torch.ones(c, device="cuda")
    layers = [DecoderLayer(DecoderAttention(a.dtype, hq, hk, d, batch, max(a.prompts) + a.tokens), random((hq + 2 * hk) * d, c), random(c, hq * d),
                           random(2 * a.hidden, c), random(c, a.hidden), ones, ones, rows=a.rows) for _ in range(a.layers)]
    embedding, head = torch.randn((a.vocab, c), device="cuda").to(dtype), Projection(random(a.vocab, c))
    limit = lambda v, t: torch.full((batch,), v, dtype=t, device="cuda")  # noqa: E731
    choice = TokenChoice(batch, a.vocab, torch.float32, limit(0.8, torch.float32), limit(50, torch.int32), limit(0.95, torch.float32), limit(0.02, torch.float32))
    last = torch.tensor(a.prompts, device="cuda").cumsum(0) - 1

    def answer(x, more):
        normed = add_norm(more, x, ones, out=a.rows)[1]
        return choice(head(normed, torch.float32), torch.rand(batch, device="cuda"))[0]

    def prompts():
        x, more = embedding[torch.randint(0, a.vocab, (sum(a.prompts),), device="cuda")], None
        for layer in layers:
            x, more = layer.prefill(x, more, a.prompts)
        return answer(x[last], more[last])

    def token(t):
        x, more = embedding[t.long()], None
        for layer in layers:
            x, more = layer.step(x, more)
        return answer(x, more)

    marks = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
    t = prompts()  # (the first calls load the kernels)
    if a.tokens:
        token(t)
    marks[0].record()
    t = prompts()
    marks[1].record()
    for _ in range(a.tokens):
        t = token(t)
    marks[2].record()
    torch.cuda.synchronize()
    print("%d layers, prompts of %s tokens: %.1f us" % (a.layers, a.prompts, marks[0].elapsed_time(marks[1]) * 1e3))
    if a.tokens:
        print("%d tokens of %d sequences: %.1f us each; the last ones: %s" % (a.tokens, batch, marks[1].elapsed_time(marks[2]) * 1e3 / a.tokens, t.tolist()))


if __name__ == "__main__":
    main()
