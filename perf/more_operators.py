"""What a decoder computes between its attention and the next token, as timed cases: the residual's addition with the root-mean-square norm, rows
written in microscaled formats (and read back), the product of such rows with weights of 4 bits, and the choice of a token.

A case is a dict of plain values.
  kind "norm": tokens, channels, residual (added first), out ("same" type, or "mx8": 8 bits with scales, read back).
  kind "rows": tokens, channels, format ("mx8", "mx4"), gate (rows of a gate and a value for each channel: silu(gate) * value is written).
  kind "product": m rows of k channels in x_format, n weights of k channels in mx4, bias.
  kind "sample": rows of vocab logits, mix: which limits the rows have ("none", "top_k", "top_p", "all"; "mixed": some of each, and greedy ones).

A microscaled matrix has rows rounded up to 32 and channels to 256.  32 channels of a row share the scale 2^(byte - 127), byte 255 no number.  mx4 codes
are E2M1, [rows / 32][channels / 32][32 rows][16 bytes], even channels in a byte's low half; mx8 codes E4M3, [rows / 32][channels / 16][32][16].
Scales are [rows / 32][channels / 256][2][32 rows][4]: the group of 32 channels 2 * i + j of eight is at [j][row][i].
"""
import math

import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
EPS = 1e-6


def _norm(dtype, tokens, channels, residual, out, **more):
    return dict(more, kind="norm", dtype=dtype, tokens=tokens, channels=channels, residual=residual, out=out)


def _rows(dtype, tokens, channels, fmt, gate, **more):
    return dict(more, kind="rows", dtype=dtype, tokens=tokens, channels=channels, format=fmt, gate=gate)


def _product(dtype, m, n, k, x_format, bias=False, **more):
    return dict(more, kind="product", dtype=dtype, m=m, n=n, k=k, x_format=x_format, bias=bias)


def _sample(dtype, rows, vocab, mix, **more):
    return dict(more, kind="sample", dtype=dtype, rows=rows, vocab=vocab, mix=mix)


def listed():
    return [
        # a decoding step of four sequences: all latency
        _norm("bf16", 4, 4096, True, "same", name="norm_bf16_t4"),
        # the packed prompts of a serving batch, on their way into the next product
        _norm("bf16", 8192, 4096, True, "mx8", name="norm_bf16_t8192"),
        # fp32, an odd number of channels, nothing to add
        _norm("f32", 1999, 1531, False, "same", name="norm_f32_t1999"),
        # the feed-forward's gated rows of a decoding step
        _rows("bf16", 16, 12288, "mx8", True, name="rows_bf16_t16"),
        # and of a batch of prompts
        _rows("bf16", 4096, 8192, "mx8", True, name="rows_bf16_t4096"),
        # fp32 weights of an odd shape are laid out
        _rows("f32", 2001, 4500, "mx4", False, name="rows_f32_t2001"),
        # one token meets a projection: the weights' way through memory
        _product("bf16", 1, 8192, 4096, "mx8", name="product_mx8_m1"),
        # the logits of a decoding batch
        _product("bf16", 32, 32000, 4096, "mx8", name="product_mx8_m32"),
        # odd sizes, fp32 results with a bias
        _product("f32", 777, 1000, 1531, "mx4", True, name="product_mx4_m777"),
        # a projection of packed prompts, 4 bits on both sides
        _product("bf16", 4096, 8192, 8192, "mx4", name="product_mx4_m4096"),
        # the next token of one conversation
        _sample("bf16", 1, 32000, "all", name="sample_bf16_r1"),
        # a serving batch whose requests ask for different things
        _sample("f32", 64, 128000, "mixed", name="sample_f32_r64"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))


def draw(rng):
    kind = rng.choice(["norm", "rows", "product", "product", "product", "sample", "sample"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "norm":
        channels = _log_int(rng, 64, 16384)
        tokens = _log_int(rng, 1, min(32768, 8192 * 4096 * 2 // (channels * SIZE[dtype])))
        out = rng.choice(["same", "same", "mx8"])
        return _norm(dtype, tokens, channels, rng.random() < 0.7, out)
    if kind == "rows":
        channels = _log_int(rng, 32, 16384)
        tokens = _log_int(rng, 1, min(32768, 4096 * 8192 * 2 // (channels * SIZE[dtype])))
        gate = rng.random() < 0.5
        return _rows(dtype, tokens, channels, "mx8" if gate else rng.choice(["mx8", "mx4"]), gate)
    if kind == "product":
        n, k = _log_int(rng, 64, 32768), _log_int(rng, 64, 16384)
        m = _log_int(rng, 1, min(8192, 4096 * 8192 * 8192 // (n * k)))
        x_format = rng.choice(["mx8", "mx4"])
        # (the matrix instruction adds products of 8-bit values less exactly than fp32 holds the result)
        return _product(dtype if x_format == "mx4" else "bf16", m, n, k, x_format, rng.random() < 0.4)
    vocab = _log_int(rng, 1000, 200000)
    rows = _log_int(rng, 1, min(256, 64 * 128000 // vocab))
    return _sample(dtype, rows, vocab, rng.choice(["none", "top_k", "top_p", "all", "mixed"]))


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _uniform(g, rows):
    return torch.rand((rows,), generator=g, device="cuda", dtype=torch.float32)


def _up(n, to):
    return (n + to - 1) // to * to


def _states(g, tokens, channels, dtype):
    """What a layer passes on: rows of different sizes, a few channels of all rows much larger than the others.  Rows begin 16 bytes apart."""
    x = _normal(g, (tokens, _up(channels, 16 // SIZE[dtype]))) * torch.exp(0.3 * _normal(g, (tokens, 1)))
    x = x * (1.0 + 20.0 * (torch.rand((1, x.shape[1]), generator=g, device="cuda") < 0.005))
    return x.to(TORCH[dtype])


def _limits(g, case):
    """Temperature, top-k, top-p, min-p and random number of every row."""
    rows, vocab, mix = case["rows"], case["vocab"], case["mix"]
    t = 0.5 + 0.9 * _uniform(g, rows)
    k = torch.exp(_uniform(g, rows) * math.log(min(vocab, 400))).round().to(torch.int32)
    p = 0.6 + 0.39 * _uniform(g, rows)
    m = 0.002 + 0.1 * _uniform(g, rows)
    which = torch.randint(0, 25, (rows,), generator=g, device="cuda")
    none = (which == 24) & (mix == "mixed")  # nothing is allowed
    which = which % 5  # 0 none, 1 top-k, 2 top-p, 3 all, 4 greedy
    if mix != "mixed":
        which = torch.full_like(which, ("none", "top_k", "top_p", "all").index(mix))
    t = torch.where(which == 4, 0.0, t)
    k = torch.where((which == 1) | (which == 3), k, 0).to(torch.int32)
    p = torch.where((which == 2) | (which == 3), p, 1.0)
    m = torch.where(which == 3, m, 0.0)
    return dict(t=t, k=k, p=p, m=m, u=_uniform(g, rows), none=none)


def prepare(case, seed):
    g, kind, t = _gen(seed), case["kind"], TORCH[case["dtype"]]
    st = dict(case=case)
    if kind == "norm":
        n, c = case["tokens"], case["channels"]
        st.update(x=_states(g, n, c, case["dtype"]), w=1.0 + 0.2 * _normal(g, (c,)))
        if case["residual"]:
            st["r"] = _states(g, n, c, case["dtype"])
            st["s"] = torch.empty_like(st["r"])
        if case["out"] == "same":
            st["y"] = torch.empty_like(st["x"])
        else:
            st.update(_empty(case["out"], n, c), y=torch.empty((n, _up(c, 8)), device="cuda", dtype=torch.bfloat16))
    elif kind == "rows":
        n, c = case["tokens"], case["channels"]
        st["x"] = _states(g, n, 2 * c if case["gate"] else c, case["dtype"])
        st.update(_empty(case["format"], n, c), y=torch.empty((n, _up(c, 8)), device="cuda", dtype=torch.bfloat16))
    elif kind == "product":
        m, n, k = case["m"], case["n"], case["k"]
        st["x"], st["xs"] = _matrix(g, _states(g, m, k, "f32")[:, :k], case["x_format"])
        st["w"], st["ws"] = _matrix(g, _normal(g, (n, k)) * k ** -0.5, "mx4")
        if case["bias"]:
            st["b"] = 0.1 * _normal(g, (n,))
        st["y"] = torch.empty((m, _up(n, 8)), device="cuda", dtype=t)
    else:
        rows, vocab = case["rows"], case["vocab"]
        x = 2.5 * _normal(g, (rows, vocab)) + 4.0 * _normal(g, (1, vocab)) * (torch.rand((1, vocab), generator=g, device="cuda") < 0.01)
        # some tokens of a row stand out, by more in one row than in another: a few share the choice, or thousands do
        x = x + 14.0 * _uniform(g, rows)[:, None] * torch.rand((rows, vocab), generator=g, device="cuda") * (
            torch.rand((rows, vocab), generator=g, device="cuda") < 40.0 / vocab)
        limits = _limits(g, case)
        # tokens that a grammar rules out: a few, or all of a row
        x = torch.where((torch.rand((rows, vocab), generator=g, device="cuda") < 0.01) | limits.pop("none")[:, None], -math.inf, x)
        st.update(limits, x=x.to(t), token=torch.empty((rows,), device="cuda", dtype=torch.int32),
                  logp=torch.empty((rows,), device="cuda", dtype=torch.float32))
    return st


def _empty(fmt, rows, channels):
    r, c = _up(rows, 32), _up(channels, 256)
    return dict(codes=torch.empty((r * c // (2 if fmt == "mx4" else 1),), device="cuda", dtype=torch.uint8),
                scales=torch.empty((r * c // 32,), device="cuda", dtype=torch.uint8))


def _matrix(g, x, fmt):
    """A microscaled matrix of the rows x in fp32; rows beyond theirs hold any bytes."""
    code, e = _quantised(_padded(x), fmt)
    c = code.shape[1]
    r = _up(x.shape[0], 32) - x.shape[0]
    if r:
        junk = lambda width: torch.randint(0, 256, (r, width), generator=g, device="cuda", dtype=torch.uint8)  # noqa: E731
        code, e = torch.cat([code, junk(c) & (15 if fmt == "mx4" else 255)]), torch.cat([e, junk(c // 32)])
    if fmt == "mx4":
        code = (code[:, 0::2] | code[:, 1::2] << 4)
    code = code.reshape(-1, 32, code.shape[1] // 16, 16).permute(0, 2, 1, 3)
    e = e.reshape(-1, 32, c // 256, 4, 2).permute(0, 2, 4, 1, 3)
    return code.reshape(-1).contiguous(), e.reshape(-1).contiguous()


# ---- the plain form -----------------------------------------------------------------------------------------------------
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _padded(x):
    """Rows in fp32, with zeros up to a multiple of 256 channels."""
    return torch.nn.functional.pad(x.float(), (0, _up(x.shape[1], 256) - x.shape[1]))


def _quantised(x, fmt):
    """Codes [rows, c] and scale exponents [rows, c / 32] of fp32 rows: the smallest power of two at which the largest of 32 rounds to 6 (mx8:
    448) at most, ties to even codes."""
    y = x.reshape(x.shape[0], -1, 32)
    top = y.abs().amax(-1).view(torch.int32)
    number = top < 0x7F800000
    e = ((top + (1 << 21)) >> 23) - 2 if fmt == "mx4" else ((top + 0x17FFFF) >> 23) - 8
    e = torch.where(number, e.clamp(min=0), 0)
    # (in two factors: the power that takes a value to its code may be beyond fp32's range)
    half = (127 - e) // 2
    power = lambda n: ((n + 127) << 23).view(torch.float32)[..., None]  # noqa: E731
    z = torch.where(number[..., None], y, 0.0) * power(half) * power(127 - e - half)
    if fmt == "mx4":
        m = z.abs()
        code = ((m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0) + 8 * torch.signbit(z)).to(torch.uint8)
    else:
        code = z.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
    return code.reshape(x.shape), torch.where(number, e, 255).to(torch.uint8)


def _values(code, e, fmt):
    """fp32 values of codes [rows, c] with scale exponents [rows, c / 32]."""
    if fmt == "mx4":
        v = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=code.device)[code.int()]
    else:
        v = code.view(torch.float8_e4m3fn).float()
    scale = torch.where(e == 255, math.nan, torch.exp2(e.float() - 127.0))
    return (v.reshape(v.shape[0], -1, 32) * scale[..., None]).reshape(v.shape)


def _decoded(codes, scales, rows, channels, fmt):
    """The fp32 values of a microscaled matrix."""
    c = _up(channels, 256)
    e = scales.reshape(-1, c // 256, 2, 32, 4).permute(0, 3, 1, 4, 2).reshape(-1, c // 32)
    if fmt == "mx4":
        b = codes.reshape(-1, c // 32, 32, 16).permute(0, 2, 1, 3).reshape(-1, c // 2)
        code = torch.stack([b & 15, b >> 4], -1).reshape(-1, c)
    else:
        code = codes.reshape(-1, c // 16, 32, 16).permute(0, 2, 1, 3).reshape(-1, c).contiguous()
    return _values(code[:rows], e[:rows], fmt)[:, :channels]


def _through(x, fmt):
    """What rows are after being written in a format."""
    code, e = _quantised(_padded(x), fmt)
    return _values(code, e, fmt)[:, :x.shape[1]].to(torch.bfloat16)


def _chosen(st):
    """In 64 bits: sums of a hundred thousand weights next to a limit decide."""
    x = st["x"].double()
    x = torch.where(torch.isnan(x), -math.inf, x)
    t, k, p, m, u = (st[name].double()[:, None] for name in "tkpmu")
    order = torch.sort(x, dim=1, descending=True, stable=True)
    top = order.values[:, :1]
    away = torch.where(order.values == top, 0.0, order.values - top)
    w = torch.exp(away / torch.where(t > 0, t, 1.0))
    w = torch.where(order.values == -math.inf, 0.0, w)
    rank = torch.arange(x.shape[1], device=x.device)[None, :]
    w = torch.where((rank < torch.where(k > 0, k, math.inf)) & ((t > 0) | (rank == 0)), w, 0.0)
    before = torch.cumsum(w, 1) - w
    kept = ((before < p * w.sum(1, keepdim=True)) | (p >= 1) | (rank == 0)) & (w >= m)
    w = torch.zeros_like(w).scatter_(1, order.indices, torch.where(kept, w, 0.0))
    run = torch.cumsum(w, 1)
    total = run[:, -1:]
    token = (run <= u * total).sum(1, keepdim=True).clamp(max=x.shape[1] - 1)
    none = top == -math.inf
    logp = torch.where(none, -math.inf, torch.log(w.gather(1, token) / total))
    return torch.where(none, -1, token)[:, 0].to(torch.int32), logp[:, 0].float()


def _plain(st):
    c = st["case"]
    t = TORCH[c["dtype"]]
    if c["kind"] == "norm":
        n = c["channels"]
        s = st["x"][:, :n].float()
        if c["residual"]:
            s = (s + st["r"][:, :n].float()).to(t).float()
        y = s * torch.rsqrt(s.square().mean(1, keepdim=True) + EPS) * st["w"]
        y = y.to(t) if c["out"] == "same" else _through(y, c["out"])
        return (s.to(t), y) if c["residual"] else y
    if c["kind"] == "rows":
        x, n = st["x"].float(), c["channels"]
        if c["gate"]:
            x = x[:, :n] * torch.sigmoid(x[:, :n]) * x[:, n:2 * n]
        return _through(x[:, :n], c["format"])
    if c["kind"] == "product":
        x, w = _decoded(st["x"], st["xs"], c["m"], c["k"], c["x_format"]), _decoded(st["w"], st["ws"], c["n"], c["k"], "mx4")
        y = torch.matmul(x, w.t())
        return (y + st["b"] if c["bias"] else y).to(t)
    return _chosen(st)


# ---- the framework's calls ----------------------------------------------------------------------------------------------
def _calls(st):
    """What a program makes once: the descriptions of its calls, and the workspace."""
    from paper_2301_01333_amd import binding

    c = st["case"]
    dt = binding.DTYPES[c["dtype"]]
    mx = {"mx4": binding.OGC_MX4, "mx8": binding.OGC_MX8}
    if c["kind"] == "norm":
        out = binding.OGC_NORM_SAME if c["out"] == "same" else binding.OGC_NORM_MX8
        wide = st["x"].stride(0)
        desc = binding.norm_desc(dt, c["tokens"], c["channels"], out, EPS, wide, st["r"].stride(0) if c["residual"] else 0,
                                 st["s"].stride(0) if c["residual"] else 0, st["y"].stride(0) if c["out"] == "same" else 0)
        if c["out"] == "same":
            return binding, desc, None
        return binding, desc, binding.mx_rows(binding.OGC_BF16, mx[c["out"]], c["tokens"], c["channels"], binding.OGC_GATE_NONE, st["y"].stride(0))
    if c["kind"] == "rows":
        gate = binding.OGC_GATE_SILU if c["gate"] else binding.OGC_GATE_NONE
        return (binding, binding.mx_rows(dt, mx[c["format"]], c["tokens"], c["channels"], gate, st["x"].stride(0)),
                binding.mx_rows(binding.OGC_BF16, mx[c["format"]], c["tokens"], c["channels"], binding.OGC_GATE_NONE, st["y"].stride(0)))
    if c["kind"] == "product":
        desc = binding.mx_product_desc(dt, mx[c["x_format"]], binding.OGC_MX4, c["m"], c["n"], c["k"], int(c["bias"]), st["y"].stride(0))
        need = binding.ogc_mx_product_workspace_bytes(desc)
    else:
        desc = binding.sample_desc(dt, c["rows"], c["vocab"], st["x"].stride(0))
        need = binding.ogc_sample_workspace_bytes(desc)
    return binding, desc, torch.empty(max(256, need), dtype=torch.uint8, device="cuda")


def _own(st):
    if "calls" not in st:
        st["calls"] = _calls(st)
    c, (binding, desc, more) = st["case"], st["calls"]
    p = lambda name: st[name].data_ptr() if name in st else 0  # noqa: E731
    stream = int(torch.cuda.current_stream().cuda_stream)
    if c["kind"] == "norm":
        same = c["out"] == "same"
        binding.ogc_norm_run(desc, p("x"), p("r"), p("w"), p("s"), p("y") if same else p("codes"), 0 if same else p("scales"), stream)
        if not same:
            binding.ogc_mx_read(more, p("codes"), p("scales"), p("y"), stream)
        y = st["y"][:, :c["channels"]]
        return (st["s"][:, :c["channels"]], y) if c["residual"] else y
    if c["kind"] == "rows":
        binding.ogc_mx_write(desc, p("x"), p("codes"), p("scales"), stream)
        binding.ogc_mx_read(more, p("codes"), p("scales"), p("y"), stream)
        return st["y"][:, :c["channels"]]
    if c["kind"] == "product":
        binding.ogc_mx_product_run(desc, p("x"), p("xs"), p("w"), p("ws"), p("b"), p("y"), more.data_ptr(), stream)
        return st["y"][:, :c["n"]]
    binding.ogc_sample_run(desc, p("x"), p("t"), p("k"), p("p"), p("m"), p("u"), p("token"), p("logp"), more.data_ptr(), stream)
    return st["token"], st["logp"]


def run(st):
    return _own(st) if own else _plain(st)


def work(case):
    """Inputs read once, outputs written once; what is read back also goes through memory as codes and scales."""
    kind, e = case["kind"], SIZE[case["dtype"]]
    held = {"mx4": 17 / 32, "mx8": 33 / 32}
    if kind in ("norm", "rows"):
        values = case["tokens"] * case["channels"]
        if kind == "rows":
            return {"bytes": values * (e * (2 if case["gate"] else 1) + 2 * held[case["format"]] + 2), "flops": values * (9 if case["gate"] else 3)}
        out = e if case["out"] == "same" else 2 * held[case["out"]] + 2
        return {"bytes": values * ((3 if case["residual"] else 1) * e + out) + 4 * case["channels"], "flops": values * 5}
    if kind == "product":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": m * k * held[case["x_format"]] + n * k * held["mx4"] + m * n * e + (4 * n if case["bias"] else 0), "flops": 2 * m * n * k}
    return {"bytes": case["rows"] * (case["vocab"] * e + 28), "flops": case["rows"] * case["vocab"] * 4}


# ---- the same results in 64 bits ----------------------------------------------------------------------------------------
def _grid(x, mantissa, largest, low):
    """In 64 bits, the nearest value of a format with so many bits behind the point, down to 2^low, and its largest value, times the group's power of two."""
    n = x.shape[1]
    y = torch.nn.functional.pad(x.double(), (0, _up(n, 32) - n)).unflatten(1, (-1, 32))
    top = y.abs().amax(-1, keepdim=True)
    emax = math.floor(math.log2(largest))
    _, e = torch.frexp(top)
    scale = torch.exp2((e - 1 - emax).double().clamp(-127, 127))
    near = lambda z: torch.exp2(torch.frexp(z.abs().clamp(min=2.0 ** low))[1].double() - 1 - mantissa)  # noqa: E731 (step at z)
    at = top / scale
    scale = torch.where((at / near(at)).round() * near(at) > largest, 2 * scale, scale)
    z = y / scale
    z = (z / near(z)).round() * near(z) * scale
    return z.flatten(1)[:, :n]


def _in_format(x, fmt):
    return _grid(x, 1, 6.0, 0) if fmt == "mx4" else _grid(x, 3, 448.0, -6)


def _held(codes, scales, rows, channels, fmt):
    """Values in 64 bits of a microscaled matrix, from the places of codes and scales."""
    c = _up(channels, 256)
    out = torch.empty((rows, channels), dtype=torch.float64, device="cuda")
    j = torch.arange(channels, device="cuda")[None, :]
    for first in range(0, rows, 1024):
        r = torch.arange(first, min(rows, first + 1024), device="cuda")[:, None]
        s = scales[r // 32 * c + j // 256 * 256 + j // 32 % 2 * 128 + r % 32 * 4 + j // 64 % 4].double()
        if fmt == "mx4":
            b = codes[r // 32 * 16 * c + j // 32 * 512 + r % 32 * 16 + j % 32 // 2].int() >> (4 * (j % 2)) & 15
            bits, expo, one, sign = b & 1, b >> 1 & 3, 2.0, b >> 3
        else:
            b = codes[r // 32 * 32 * c + j // 16 * 512 + r % 32 * 16 + j % 16].int()
            bits, expo, one, sign = b & 7, b >> 3 & 15, 8.0, b >> 7
        bias = 1 if fmt == "mx4" else 7
        v = torch.where(expo == 0, bits / one, 1 + bits / one) * torch.exp2(expo.clamp(min=1).double() - bias)
        out[first:first + 1024] = torch.where(sign == 1, -v, v) * torch.exp2(s - 127.0)
    return out


def _picked(x, t, k, p, m, u):
    """One row in 64 bits: its logits that are kept, from the largest down, then the choice among them in their own order."""
    if not (x > -math.inf).any():
        return -1, -math.inf
    if not t > 0:
        return int((x == x.max()).nonzero()[0, 0]), 0.0
    order = torch.argsort(-x, stable=True)
    logs = (x[order] - x.max()) / t
    if k > 0:
        logs, order = logs[:k], order[:k]
    share = torch.softmax(logs, 0)
    if p < 1:
        n = max(1, int((torch.cumsum(share, 0) - share < p).sum()))
        share, order, logs = share[:n], order[:n], logs[:n]
    keep = logs >= math.log(m) if m > 0 else logs > -math.inf
    order, logs = order[keep], logs[keep]
    order, at = torch.sort(order)
    share = torch.cumsum(torch.softmax(logs[at], 0), 0)
    i = min(int((share <= u * share[-1]).sum()), len(order) - 1)
    return int(order[i]), float(torch.log_softmax(logs[at], 0)[i])


def exact(case, seed):
    st, kind = prepare(case, seed), case["kind"]
    if kind == "norm":
        n = case["channels"]
        s = st["x"][:, :n].double()
        if case["residual"]:
            s = (s + st["r"][:, :n].double()).to(TORCH[case["dtype"]]).double()
        y = s / torch.sqrt((s ** 2).mean(1, keepdim=True) + EPS) * st["w"].double()
        y = y if case["out"] == "same" else _in_format(y, case["out"])
        return (s, y) if case["residual"] else y
    if kind == "rows":
        x, n = st["x"].double(), case["channels"]
        if case["gate"]:
            x = x[:, :n] / (1 + torch.exp(-x[:, :n])) * x[:, n:2 * n]
        return _in_format(x[:, :n], case["format"])
    if kind == "product":
        w = _held(st["w"], st["ws"], case["n"], case["k"], "mx4")
        y = torch.matmul(_held(st["x"], st["xs"], case["m"], case["k"], case["x_format"]), w.t())
        return y + st["b"].double() if case["bias"] else y
    x = torch.nan_to_num(st["x"].double(), nan=-math.inf, neginf=-math.inf)
    limits = [st[name].tolist() for name in "tkpmu"]
    got = [_picked(x[r], *(v[r] for v in limits)) for r in range(case["rows"])]
    return torch.tensor([g[0] for g in got], dtype=torch.int32), torch.tensor([g[1] for g in got], dtype=torch.float64)
