"""The operators of a decoder's attention block as timed cases: head norms with rotary positions, the key/value cache held in
4 bits (written and read back), attention over that cache, attention over packed prompts.

A case is a dict of plain values.
  kind "rope": tokens, q_heads, kv_heads, head_dim, rot (rotated channels), layout ("half", "interleaved"), norm, far (positions
    reach it), stretch (divisor of the frequencies).
  kind "store": batch sequences with up to `held` tokens in the cache get up to `fresh` new ones each; all of them are read back.
  kind "step": batch sequences of up to `longest` cached tokens, the last `fresh` of which ask.
  kind "prompt": batch sequences of up to `longest` new tokens, up to `earlier` keys of each before them.
`even`: every sequence is as long as the longest; otherwise lengths spread from 1 to it.  page: tokens of a cache page.

A cache is uint8 [pages][kv heads][page / 32][34 * head_dim]: for 32 tokens of a head the 4-bit codes of the keys [32][d / 2], those
of the values [d / 32][token / 8][channel % 16][channel / 16 % 2][token % 8 / 2], and the scales' exponents, [d / 32][32] for keys and then
values.  Even channels (values: even tokens) are in a byte's low half.  A code is E2M1, a scale 2^(byte - 127), byte 255 no number.
"""
import math

import numpy as np
import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
EPS = 1e-6


def _rope(dtype, tokens, q_heads, kv_heads, head_dim, rot, layout="half", norm=True, far=8192, stretch=1.0, **more):
    return dict(more, kind="rope", dtype=dtype, tokens=tokens, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, rot=rot,
                layout=layout, norm=norm, far=far, stretch=stretch)


def _store(dtype, batch, held, fresh, kv_heads, head_dim, page=64, even=False, **more):
    return dict(more, kind="store", dtype=dtype, batch=batch, held=held, fresh=fresh, kv_heads=kv_heads, head_dim=head_dim, page=page,
                even=even)


def _step(dtype, batch, longest, q_heads, kv_heads, head_dim, fresh=1, page=64, even=False, **more):
    return dict(more, kind="step", dtype=dtype, batch=batch, longest=longest, fresh=fresh, q_heads=q_heads, kv_heads=kv_heads,
                head_dim=head_dim, page=page, even=even)


def _prompt(dtype, batch, longest, q_heads, kv_heads, head_dim, earlier=0, even=False, **more):
    return dict(more, kind="prompt", dtype=dtype, batch=batch, longest=longest, earlier=earlier, q_heads=q_heads, kv_heads=kv_heads,
                head_dim=head_dim, even=even)


def listed():
    return [
        # one decoding step of eight sequences: all latency
        _rope("bf16", 8, 32, 8, 128, 128, name="rope_bf16_t8"),
        # the packed prompts of a serving batch
        _rope("bf16", 8192, 32, 8, 128, 128, name="rope_bf16_t8192"),
        # fp32, half of the head rotated in interleaved pairs, no norms, positions of a context stretched to a million
        _rope("f32", 1999, 16, 16, 96, 48, "interleaved", False, 1 << 20, 4.0, name="rope_f32_t1999"),
        # a decoding step appends one token to sixteen short conversations; everything they hold is read back
        _store("bf16", 16, 250, 1, 8, 128, name="store_bf16_b16"),
        # chunks of prompts enter the cache behind what it holds, at odd places
        _store("bf16", 8, 301, 1999, 8, 128, name="store_bf16_b8"),
        # one conversation of a thousand tokens: latency
        _step("bf16", 1, 1000, 32, 8, 128, name="step_bf16_s1000_b1"),
        # an ordinary serving batch, lengths all different
        _step("bf16", 32, 4001, 32, 8, 128, name="step_bf16_s4001_b32"),
        # the largest batch at its full context
        _step("bf16", 64, 8192, 32, 8, 128, even=True, name="step_bf16_s8192_b64"),
        # four proposed tokens at a time are checked, one key head for each query head, fp32
        _step("f32", 12, 1531, 12, 12, 64, fresh=4, page=32, name="step_f32_s1531_b12"),
        # one short odd prompt, one key head for each query head
        _prompt("bf16", 1, 197, 12, 12, 64, name="prompt_bf16_s197"),
        # prompts of all lengths packed into one call, grouped heads
        _prompt("bf16", 8, 4096, 32, 8, 128, name="prompt_bf16_s4096_b8"),
        # fp32 chunks behind earlier keys
        _prompt("f32", 4, 700, 16, 4, 96, earlier=333, name="prompt_f32_s700_b4"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rope", "store", "step", "step", "prompt", "prompt"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    d, kv = rng.choice([32, 64, 96, 128, 128]), rng.choice([1, 2, 4, 8, 12])
    heads = kv * rng.choice([1, 2, 3, 4, 8])
    even = rng.random() < 0.3
    if kind == "rope":
        most = int(8192 * 40 * 128 * 2 / ((heads + kv) * d * SIZE[dtype]))
        rot = rng.choice([d, d, d // 2, d // 4])
        return _rope(dtype, _log_int(rng, 1, min(32768, most)), heads, kv, d, rot, rng.choice(["half", "interleaved"]), rng.random() < 0.6,
                     _log_int(rng, 4096, 1 << 20), rng.choice([1.0, 1.0, 4.0, 8.0]))
    page = rng.choice([32, 64, 128, 256])
    if kind == "store":
        batch = _log_int(rng, 1, 64)
        most = int(8 * 2300 * 8 * 128 * 2 / (batch * kv * d * SIZE[dtype]))
        fresh = _log_int(rng, 1, max(1, min(4096, most)))
        held = _log_int(rng, 1, max(1, min(2048, most - fresh + 1)))
        return _store(dtype, batch, held, fresh, kv, d, page, even)
    if kind == "step":
        fresh = rng.choice([1, 1, 1, 2, 3, 5])
        batch = _log_int(rng, 1, 64)
        most = int(64 * 8192 * 32 * 128 / (batch * max(heads, 2 * kv) * d * fresh * (1 if dtype == "bf16" else 2)))
        return _step(dtype, batch, max(fresh, _log_int(rng, 16, max(16, min(32768, most)))), heads, kv, d, fresh, page, even)
    batch = _log_int(rng, 1, 16)
    most = 8 * 4096 * 4096 * 32 / (batch * heads * (1 if dtype == "bf16" else 8))
    longest = _log_int(rng, 1, max(1, min(8192, int(math.sqrt(most)))))
    earlier = 0 if rng.random() < 0.6 else int(rng.uniform(0, max(0.0, most / longest - longest)) / 4)
    return _prompt(dtype, batch, longest, heads, kv, d, min(earlier, 4000), even)


# ---- lengths: whole numbers that the case alone decides -----------------------------------------------------------------
def _spread(count, longest, even, phase=0.0):
    """`count` lengths from 1 to `longest`, the first the longest, spread evenly and in no order."""
    if even:
        return [longest] * count
    return [longest] + [1 + int((longest - 1) * ((0.6180339887 * i + phase) % 1.0)) for i in range(1, count)]


def _lengths(case):
    """(new tokens, all tokens) of every sequence."""
    if case["kind"] == "step":
        total = [max(n, case["fresh"]) for n in _spread(case["batch"], case["longest"], case["even"])]
        return [case["fresh"]] * case["batch"], total
    fresh = _spread(case["batch"], case["fresh"] if case["kind"] == "store" else case["longest"], case["even"])
    before = case["held"] if case["kind"] == "store" else case["earlier"]
    before = _spread(case["batch"], before, case["even"], 0.3) if before else [0] * case["batch"]
    return fresh, [a + b for a, b in zip(fresh, before)]


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _heads(g, tokens, heads, d, dtype, loud=False):
    """What a projection leaves of a tensor's heads; `loud`: a few channels of every head are much larger, as keys' are."""
    x = _normal(g, (tokens, heads, d))
    if loud:
        x = x * (1.0 + 5.0 * (torch.rand((1, heads, d), generator=g, device="cuda") < 0.04))
    return x.to(TORCH[dtype])


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _sums(values):
    return _ints([0] + np.cumsum(values).tolist())


def _frequencies(case):
    i = np.arange(0, case["rot"], 2, dtype=np.float64)
    return torch.from_numpy(10000.0 ** (-i / case["rot"]) / case["stretch"]).cuda()


def _table(g, case, total):
    """A page table in no order, -1 beyond a sequence's pages, and the number of pages."""
    page = case["page"]
    pages = [(n + page - 1) // page for n in total]
    order = torch.randperm(sum(pages) + 3, generator=g, device="cuda").to(torch.int32)
    at = torch.arange(max(pages), device="cuda")[None, :]
    first = _sums(pages)[:-1, None].long()
    used = at < _ints(pages)[:, None]
    table = torch.where(used, order[(first + at).clamp(max=sum(pages) - 1)], -1).to(torch.int32).contiguous()
    return table, sum(pages) + 3


def _cache(g, case, total):
    """A cache as it stands after `total` tokens of every sequence were written; what no token was written to is any bytes."""
    h, d, page = case["kv_heads"], case["head_dim"], case["page"]
    table, pages = _table(g, case, total)
    cache = torch.randint(0, 256, (pages, h, page // 32, 34 * d), generator=g, device="cuda", dtype=torch.uint8)
    kc, vc, ks, vs = _codes(cache)
    where = _where(table, page, _ints(total))
    n = sum(total)
    (a, s), (b, t) = (_quantised(_heads(g, n, h, d, case["dtype"], loud).float()) for loud in (True, False))
    kc[where], vc[where], ks[where], vs[where] = a, b, s, t
    return _bytes(kc, vc, ks, vs, page), table


def prepare(case, seed):
    g, d, t = _gen(seed), case["head_dim"], TORCH[case["dtype"]]
    st = dict(case=case, d=d)
    if case["kind"] == "rope":
        n, hq, hk = case["tokens"], case["q_heads"], case["kv_heads"]
        qkv = _heads(g, n, hq + 2 * hk, d, case["dtype"])  # one buffer, as one projection leaves it
        st.update(q=qkv[:, :hq], k=qkv[:, hq:hq + hk], freq=_frequencies(case),
                  pos=torch.randint(0, case["far"], (n,), generator=g, device="cuda", dtype=torch.int32),
                  qw=1.0 + 0.2 * _normal(g, (d,)), kw=1.0 + 0.2 * _normal(g, (d,)),
                  qo=torch.empty((n, hq, d), device="cuda", dtype=t), ko=torch.empty((n, hk, d), device="cuda", dtype=t))
        return st
    fresh, total = _lengths(case)
    n = sum(fresh)
    st.update(cu=_sums(fresh), max_fresh=max(fresh), max_total=max(total))
    if case["kind"] == "prompt":
        hq, hk, m = case["q_heads"], case["kv_heads"], sum(total)
        st.update(q=_heads(g, n, hq, d, case["dtype"]), k=_heads(g, m, hk, d, case["dtype"], True),
                  v=_heads(g, m, 2 * hk, d, case["dtype"])[:, hk:], cu_k=_sums(total), o=torch.empty((n, hq, d), device="cuda", dtype=t))
        return st
    st["cache"], st["table"] = _cache(g, case, total)
    st["lens"] = _ints(total)
    if case["kind"] == "step":
        hq = case["q_heads"]
        st.update(q=_heads(g, n, hq, d, case["dtype"]), o=torch.empty((n, hq, d), device="cuda", dtype=t))
        return st
    h, m = case["kv_heads"], sum(total)
    st.update(k=_heads(g, n, h, d, case["dtype"], True), v=_heads(g, n, 2 * h, d, case["dtype"])[:, h:],
              start=_ints([a - b for a, b in zip(total, fresh)]), cu_all=_sums(total), zero=torch.zeros_like(st["lens"]), rows=m,
              ko=torch.empty((m, h, d), device="cuda", dtype=t), vo=torch.empty((m, h, d), device="cuda", dtype=t))
    return st


# ---- the plain form -----------------------------------------------------------------------------------------------------
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _quantised(x):
    """Codes [..., d] and scale exponents [..., d / 32] of fp32 values: the largest of 32 rounds to 6 at most, ties to even codes."""
    y = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    e = (((y.abs().amax(-1).view(torch.int32) + (1 << 21)) >> 23) - 2).clamp(0, 252)
    m = y.abs() * ((254 - e) << 23).view(torch.float32)[..., None]
    code = ((m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0)
            + 8 * torch.signbit(y)).to(torch.uint8)
    return code.reshape(x.shape), e.to(torch.uint8)


def _values(code, e):
    """fp32 values of codes [..., d] with scale exponents [..., d / 32]."""
    lut = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=code.device)
    scale = torch.where(e == 255, math.nan, torch.exp2(e.float() - 127.0))
    return lut[code.int()] * scale.repeat_interleave(32, -1)


def _halves(b):
    return torch.stack([b & 15, b >> 4], -1)


def _codes(cache):
    """Codes and exponents of a whole cache as [pages * page, heads, ...]: keys, values, the keys' exponents, the values'."""
    p, h, nb, rec = cache.shape
    d = rec // 34
    tokens_first = lambda x: x.permute(0, 2, 3, 1, 4).reshape(p * nb * 32, h, x.shape[-1]).contiguous()  # noqa: E731
    kc = _halves(cache[..., :16 * d].reshape(p, h, nb, 32, d // 2)).reshape(p, h, nb, 32, d)
    vc = _halves(cache[..., 16 * d:32 * d].reshape(p, h, nb, d // 32, 4, 16, 2, 4))
    vc = vc.permute(0, 1, 2, 4, 7, 8, 3, 6, 5).reshape(p, h, nb, 32, d)
    ks, vs = (cache[..., a * d:(a + 1) * d].reshape(p, h, nb, d // 32, 32).transpose(3, 4) for a in (32, 33))
    return tokens_first(kc), tokens_first(vc), tokens_first(ks), tokens_first(vs)


def _bytes(kc, vc, ks, vs, page):
    """The cache that _codes() takes apart."""
    n, h, d = kc.shape
    blocks = lambda x: x.reshape(n // page, page // 32, 32, h, x.shape[-1]).permute(0, 3, 1, 2, 4)  # noqa: E731
    flat = lambda x: x.reshape(n // page, h, page // 32, -1)  # noqa: E731
    kc = blocks(kc).reshape(n // page, h, page // 32, 32, d // 2, 2)
    vc = blocks(vc).reshape(n // page, h, page // 32, 4, 4, 2, d // 32, 2, 16).permute(0, 1, 2, 6, 3, 8, 7, 4, 5)
    return torch.cat([flat(kc[..., 0] | kc[..., 1] << 4), flat(vc[..., 0] | vc[..., 1] << 4), flat(blocks(ks).transpose(3, 4)),
                      flat(blocks(vs).transpose(3, 4))], -1).contiguous()


def _where(table, page, lens, start=None):
    """Places in [pages * page] of the tokens start .. lens - 1 of every sequence, one sequence after the other."""
    j = torch.arange(table.shape[1] * page, device=table.device)[None, :]
    at = table.long().clamp(min=0).repeat_interleave(page, 1) * page + j % page
    keep = j < lens[:, None]
    return at[keep if start is None else keep & (j >= start[:, None])]


def _attended(q, k, v, visible, scale):
    """q [b, n, hq, d], k and v [b, m, hk, d] in fp32, visible [b, n, m] -> [b, n, hq, d]; a row that sees nothing gives zeros."""
    b, n, hq, d = q.shape
    hk = k.shape[2]
    q = q.reshape(b, n, hk, hq // hk, d).permute(0, 2, 3, 1, 4).reshape(b, hk, hq // hk * n, d)
    s = (torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()) * scale).reshape(b, hk, hq // hk, n, -1)
    s = s.masked_fill(~visible[:, None, None], -math.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=-3e38))
    o = torch.matmul(p.reshape(b, hk, hq // hk * n, -1), v.permute(0, 2, 1, 3).contiguous()).reshape(b, hk, hq // hk, n, d)
    total = p.sum(-1, keepdim=True)
    return (o / torch.where(total == 0, 1.0, total)).permute(0, 3, 1, 2, 4).reshape(b, n, hq, d)


def _padded(x, cu, longest):
    """Packed rows [tokens, h, d] as [sequences, longest, h, d] in fp32, zeros beyond a sequence, and which rows are its own."""
    at = torch.arange(longest, device=x.device)[None, :]
    inside = at < (cu[1:] - cu[:-1])[:, None]
    rows = (cu[:-1, None].long() + at).clamp(max=x.shape[0] - 1)
    return torch.where(inside[..., None, None], x[rows].float(), 0.0), inside


def _visible(q_lens, k_lens, n, m):
    i, j = torch.arange(n, device="cuda")[None, :, None], torch.arange(m, device="cuda")[None, None, :]
    return j <= i + (k_lens - q_lens)[:, None, None]


def _rotated(st, x, w):
    c = st["case"]
    x = x.float()
    if c["norm"]:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w
    angle = st["pos"].double()[:, None, None] * st["freq"]
    cos, sin = angle.cos().float(), angle.sin().float()
    r = c["rot"]
    if c["layout"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos, x[..., r:]], -1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), x[..., r:]], -1)
    return y.to(TORCH[c["dtype"]])


def _plain(st):
    c = st["case"]
    t = TORCH[c["dtype"]]
    if c["kind"] == "rope":
        return _rotated(st, st["q"], st["qw"]), _rotated(st, st["k"], st["kw"])
    fresh = st["cu"][1:] - st["cu"][:-1]
    if c["kind"] == "prompt":
        (q, mine), (k, _), (v, _) = (_padded(x, cu, n) for x, cu, n in (
            (st["q"], st["cu"], st["max_fresh"]), (st["k"], st["cu_k"], st["max_total"]), (st["v"], st["cu_k"], st["max_total"])))
        visible = _visible(fresh, st["cu_k"][1:] - st["cu_k"][:-1], st["max_fresh"], st["max_total"])
        return _attended(q, k, v, visible, c["head_dim"] ** -0.5)[mine].to(t)
    if c["kind"] == "step":
        p, h, nb, rec = st["cache"].shape
        b, m = st["table"].shape
        kc, vc, ks, vs = (x.reshape(b, m * nb * 32, h, -1) for x in _codes(st["cache"][st["table"].long().clamp(min=0)].flatten(0, 1)))
        held = torch.arange(m * nb * 32, device="cuda")[None, :] < st["lens"][:, None]
        k, v = (torch.where(held[..., None, None], _values(x, e), 0.0) for x, e in ((kc, ks), (vc, vs)))
        q, mine = _padded(st["q"], st["cu"], st["max_fresh"])
        return _attended(q, k, v, _visible(fresh, st["lens"], st["max_fresh"], m * nb * 32), c["head_dim"] ** -0.5)[mine].to(t)
    kc, vc, ks, vs = _codes(st["cache"])
    new = _where(st["table"], c["page"], st["lens"], st["start"])
    kc[new], ks[new] = _quantised(st["k"].float())
    vc[new], vs[new] = _quantised(st["v"].float())
    st["cache"].copy_(_bytes(kc, vc, ks, vs, c["page"]))
    every = _where(st["table"], c["page"], st["lens"])
    return _values(kc[every], ks[every]).to(t), _values(vc[every], vs[every]).to(t)


# ---- the framework's calls ----------------------------------------------------------------------------------------------
def _calls(st):
    """What a program makes once: the descriptions of its calls, and the workspace."""
    from paper_2301_01333_amd import binding

    c = st["case"]
    dt, d = binding.DTYPES[c["dtype"]], c["head_dim"]
    two = lambda x: x.stride()[:2]  # noqa: E731
    if c["kind"] == "rope":
        return binding, binding.rope_desc(
            dt, c["tokens"], c["q_heads"], c["kv_heads"], d, c["rot"],
            binding.OGC_ROPE_HALF if c["layout"] == "half" else binding.OGC_ROPE_INTERLEAVED, int(c["norm"]), EPS, 1.0,
            two(st["q"]), two(st["k"]), two(st["qo"]), two(st["ko"]))
    if c["kind"] == "prompt":
        return binding, binding.prompt_desc(
            dt, c["batch"], c["q_heads"], c["kv_heads"], d, st["q"].shape[0], st["k"].shape[0], st["max_fresh"], st["max_total"],
            d ** -0.5, 1, two(st["q"]), two(st["k"]), two(st["v"]), two(st["o"]))
    cache = binding.kv4_desc(c["kv_heads"], d, c["page"], st["cache"].shape[0], c["batch"], st["table"].shape[1])
    if c["kind"] == "store":
        return (binding, cache, binding.kv4_rows(dt, st["k"].shape[0], st["max_fresh"], two(st["k"]), two(st["v"])),
                binding.kv4_rows(dt, st["rows"], st["max_total"], two(st["ko"]), two(st["vo"])))
    asks = binding.kv4_attention_desc(dt, c["q_heads"], st["q"].shape[0], st["max_fresh"], st["max_total"], d ** -0.5, two(st["q"]),
                                      two(st["o"]))
    space = torch.empty(max(256, binding.ogc_kv4_attention_workspace_bytes(cache, asks)), dtype=torch.uint8, device="cuda")
    return binding, cache, asks, space


def _own(st):
    if "calls" not in st:
        st["calls"] = _calls(st)
    kind, calls = st["case"]["kind"], st["calls"]
    binding = calls[0]
    p = lambda name: st[name].data_ptr()  # noqa: E731
    stream = int(torch.cuda.current_stream().cuda_stream)
    if kind == "rope":
        binding.ogc_rope_run(calls[1], p("q"), p("k"), p("qw"), p("kw"), p("pos"), p("freq"), p("qo"), p("ko"), stream)
        return st["qo"], st["ko"]
    if kind == "prompt":
        binding.ogc_prompt_run(calls[1], p("q"), p("k"), p("v"), p("cu"), p("cu_k"), p("o"), stream)
        return st["o"]
    if kind == "step":
        binding.ogc_kv4_attention_run(calls[1], calls[2], p("q"), p("cu"), p("lens"), p("table"), p("cache"), p("o"), calls[3].data_ptr(),
                                      stream)
        return st["o"]
    binding.ogc_kv4_write(calls[1], calls[2], p("k"), p("v"), p("cu"), p("start"), p("table"), p("cache"), stream)
    binding.ogc_kv4_read(calls[1], calls[3], p("cache"), p("cu_all"), p("zero"), p("table"), p("ko"), p("vo"), stream)
    return st["ko"], st["vo"]


def run(st):
    return _own(st) if own else _plain(st)


def work(case):
    """Inputs read once, outputs written once; keys that no query sees, and scores, count nothing."""
    e, d = SIZE[case["dtype"]], case["head_dim"]
    if case["kind"] == "rope":
        values = case["tokens"] * (case["q_heads"] + case["kv_heads"]) * d
        return {"bytes": 2 * values * e + 4 * case["tokens"] + 4 * case["rot"] + (8 * d if case["norm"] else 0),
                "flops": values * (7 if case["norm"] else 3)}
    fresh, total = _lengths(case)
    kv = 2 * case["kv_heads"] * d
    if case["kind"] == "store":  # new values in, their codes out; all codes in, all values out
        return {"bytes": sum(fresh) * kv * (e + 17 / 32) + sum(total) * kv * (e + 17 / 32), "flops": sum(fresh) * kv * 4 + sum(total) * kv}
    pairs = sum(n * m - n * (n - 1) // 2 for n, m in zip(fresh, total))
    q = 2 * sum(fresh) * case["q_heads"] * d * e
    return {"bytes": q + sum(total) * kv * (17 / 32 if case["kind"] == "step" else e), "flops": 4 * pairs * case["q_heads"] * d}


# ---- the same results in 64 bits ----------------------------------------------------------------------------------------
def _softmax_sum(q, k, v):
    """One sequence in 64 bits: q [n, hq, d], k and v [m, hk, d]; query i sees the keys up to i + m - n."""
    n, m, group = q.shape[0], k.shape[0], q.shape[1] // k.shape[1]
    out = torch.zeros_like(q)
    later = torch.arange(m, device=q.device)[None, :] > torch.arange(n, device=q.device)[:, None] + (m - n)
    for h in range(q.shape[1]):
        s = q[:, h].contiguous() @ k[:, h // group].t().contiguous() / math.sqrt(q.shape[2])
        w = torch.softmax(s.masked_fill(later, -math.inf), 1)
        out[:, h] = torch.nan_to_num(w) @ v[:, h // group].contiguous()
    return out


def _held(cache, pages, head_dim, count, which):
    """Values in 64 bits of tokens 0 .. count - 1 on the given pages, from the places of their codes and exponents; which: 0 keys, 1 values."""
    d, nb = head_dim, cache.shape[2]
    t, c = torch.arange(count, device="cuda")[:, None], torch.arange(d, device="cuda")[None, :]
    page, block, r = pages.long()[t // (32 * nb)], t // 32 % nb, t % 32
    if which == 0:
        at, high = r * (d // 2) + c // 2, c % 2
    else:
        at, high = 16 * d + c // 32 * 512 + r // 8 * 128 + c % 16 * 8 + c // 16 % 2 * 4 + r % 8 // 2, r % 2
    flat = cache.permute(0, 2, 1, 3)  # page, block, head, byte
    code = (flat[page, block, :, at].int() >> (4 * high[..., None])) & 15
    e = flat[page, block, :, (32 + which) * d + c // 32 * 32 + r].double()
    mag = code & 7
    value = torch.where(mag < 2, mag / 2.0, (2.0 + mag % 2) * torch.exp2((mag // 2 - 2).double()))
    return (torch.where(code > 7, -value, value) * torch.exp2(e - 127.0)).transpose(1, 2)  # token, head, channel


def _rounded(x):
    """What the cache holds of x, in 64 bits: steps of 1/2 up to 2, of 1 up to 4 and of 2 up to 6 times the group's power of two."""
    y = x.double().unflatten(-1, (-1, 32))
    top = y.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top)  # top = m * 2^e, m in [1/2, 1): up to 7 times the power rounds to 6, from 7 on it would be 8
    power = torch.exp2((e - 3 + (m >= 0.875).int()).double().clamp(-127, 125))
    z = y.abs() / power
    step = torch.where(z < 2, 0.5, torch.where(z < 4, 1.0, 2.0))
    return (torch.sign(y) * ((z / step).round() * step).clamp(max=6.0) * power).flatten(-2)


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "rope":
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), st["pos"].double()[:, None] * st["freq"])[:, None]
        outs = []
        for x, w in ((st["q"], st["qw"]), (st["k"], st["kw"])):
            x = x.double()
            if case["norm"]:
                x = x / torch.sqrt((x ** 2).mean(-1, keepdim=True) + EPS) * w.double()
            head, tail = x[..., :case["rot"]], x[..., case["rot"]:]
            z = torch.complex(*(y.contiguous() for y in (head.chunk(2, -1) if case["layout"] == "half" else head.unflatten(-1, (-1, 2)).unbind(-1)))) * turn
            head = torch.cat([z.real, z.imag], -1) if case["layout"] == "half" else torch.view_as_real(z).flatten(-2)
            outs.append(torch.cat([head, tail], -1))
        return tuple(outs)
    fresh, total = _lengths(case)
    first, outs = 0, []
    for b, (n, m) in enumerate(zip(fresh, total)):
        if case["kind"] == "prompt":
            at = sum(total[:b])
            outs.append(_softmax_sum(st["q"][first:first + n].double(), st["k"][at:at + m].double(), st["v"][at:at + m].double()))
        else:
            k, v = (_held(st["cache"], st["table"][b], case["head_dim"], m, which) for which in (0, 1))
            if case["kind"] == "step":
                outs.append(_softmax_sum(st["q"][first:first + n].double(), k, v))
            else:
                k[m - n:], v[m - n:] = _rounded(st["k"][first:first + n]), _rounded(st["v"][first:first + n])
                outs.append((k, v))
        first += n
    return tuple(torch.cat(x) for x in zip(*outs)) if case["kind"] == "store" else torch.cat(outs)
