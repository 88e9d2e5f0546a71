"""The decoder's attention block at the ends of what its inputs may be: the largest and smallest values, queries and lengths.  Oracle and
tolerances: test_gpu_decoder.py."""
import numpy as np
import pytest

from oracle import decoder
from paper_2301_01333_amd import binding
from test_gpu_decoder import Paged, dt, empty, inside, ints, rows_of, stream, sums, tolerance, torch_, two, untouched
from test_gpu_decoder_kernels import WIDE, prompts, streams

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("qs,ks,causal", [([1], [33], 1), ([3], [33], 0), ([1, 70, 31], [1, 95, 63], 0), ([2, 40], [66, 129], 1)])
def test_prompt_infinite_last_values(dtype, d, many, qs, ks, causal):
    """A block of keys ends inside a unit, and the last value that there is holds infinities: they are the results of the rows that see it, and what
    follows the last key adds nothing to them."""
    torch = torch_()
    last = np.cumsum(ks) - 1

    def spoil(q, k, v):
        v[last, :, 3], v[last, :, d - 1] = float("inf"), float("-inf")

    kernel = "ogc_prompt_split_kernel<%d>" % (d // 32) if dtype == "f32" else streams(d) if many else "ogc_prompt_few_kernel<%d>" % (d // 32)
    o = prompts(kernel, dtype, qs, ks, 4, 2, d, d + sum(ks), causal=causal, spoil=spoil, copies=16 if many and dtype == "f32" else None)
    at = 0
    for a in qs:
        seen = o[at:at + a] if not causal else o[at + a - 1:at + a]
        assert (seen[..., 3] == float("inf")).all() and (seen[..., d - 1] == float("-inf")).all()
        assert torch.isfinite(o[at:at + a, :, 4:d - 1]).all() and (not causal or torch.isfinite(o[at:at + a - 1]).all())
        at += a


# ---- attention over the cache -----------------------------------------------------------------------------------------------
def ask(dtype, c, q, fresh, lens, scale, shared):
    """What the queries q get; shared: whether several workgroups have a sequence."""
    torch = torch_()
    n, hq, d = q.shape
    raw, o = empty(n, hq, d, dtype)
    cu, ln = sums(fresh), ints(lens)
    desc = binding.kv4_attention_desc(binding.DTYPES[dtype], hq, n, max(fresh), max(lens), scale, two(q), two(o))
    need = binding.ogc_kv4_attention_workspace_bytes(c.desc, desc)
    assert (need > 0) == shared
    ws = torch.full((max(16, need),), 0xFF, dtype=torch.uint8, device="cuda")
    binding.ogc_kv4_attention_run(c.desc, desc, q.data_ptr(), cu.data_ptr(), ln.data_ptr(), c.table.data_ptr(), c.device.data_ptr(), o.data_ptr(), ws.data_ptr(), stream())
    torch.cuda.synchronize()
    assert untouched(raw)
    return o


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shared", [True, False])
@pytest.mark.parametrize("d,late", [(64, False), (96, True), (128, True)])
def test_step_sums_of_the_largest_values(dtype, shared, d, late):
    """Thousands of values near the largest that there is have a finite mean, whatever their sum is; channels of the smallest ones beside them keep their
    digits.  late: the scores grow slowly, so that the weights are above those that their reference has."""
    torch = torch_()
    rng = np.random.default_rng(d)
    n, heads, batch = 4000, 2, 1
    if not shared:  # enough workgroups without splits
        heads, batch = 8, 96
    lens = [n] + [1 + i % 5 for i in range(batch - 1)]
    print("case: largest values", dtype, shared, d, late, flush=True)
    c = Paged(rng, lens, heads, d, 64)
    data = c.oracle.data
    data[..., :16 * d] = rng.integers(0, 256, data[..., :16 * d].shape)
    data[..., 16 * d:32 * d] = rng.integers(0, 256, data[..., 16 * d:32 * d].shape) & 0x77 | 0x44   # 2 .. 6, all above zero
    data[..., 32 * d:33 * d] = 122
    data[..., 33 * d:33 * d + 32] = 252          # 2^125 ..
    data[..., 33 * d + 32:34 * d] = 5            # ... and 2^-122
    if late:  # channel 0 of the keys is the only one, and grows over sixteen pages, a wavefront's share
        data[..., :16 * d] = 0
        for e in range(c.rows.shape[1]):
            for b in range(batch):
                if c.rows[b, e] >= 0:
                    data[c.rows[b, e], :, :, 0:16 * d:d // 2] = 2
                    data[c.rows[b, e], :, :, 32 * d:32 * d + 32] = 126 + e % 16 // 4
    c.device.copy_(torch.from_numpy(data))
    q, q64 = rows_of(rng, batch, heads, d, dtype, "plain", 0.5)
    if late:
        q.fill_(10.0)
        q64 = q.double().cpu().numpy()
    o = ask(dtype, c, q, [1] * batch, lens, 0.125, shared)
    for b, m in enumerate(lens[:4]):
        k, v, _ = c.tokens(b, m)
        want = decoder.attend(q64[b:b + 1], k, v, np.ones((1, m), dtype=bool), 0.125)
        assert np.isfinite(want[0]).all()
        inside(o[b:b + 1], want[0], tolerance(dtype, *want, m, d), "sequence %d" % b)


@pytest.mark.parametrize("shared", [True, False])
@pytest.mark.parametrize("size,byte,scale", [(2.0 ** -120, 246, 0.125), (2.0 ** -146, 252, 2.0 ** 18), (2.0 ** 64, 63, 0.125), (3.402e38, 2, 2.0 ** -5)])
def test_step_small_and_large_fp32_queries(shared, size, byte, scale):
    """Queries at both ends of fp32 whose scores are ordinary, as the keys are at the other end: all their digits count."""
    torch = torch_()
    rng = np.random.default_rng(byte)
    d, hk, hq = 96, 2, 4
    lens = [1500, 40, 7] if shared else [300, 40, 7]
    print("case: queries of", size, shared, flush=True)
    c = Paged(rng, lens, hk, d, 64)
    c.oracle.data[..., 32 * d:33 * d] = byte
    c.oracle.data[..., 33 * d:34 * d] = 127
    c.device.copy_(torch.from_numpy(c.oracle.data))
    x = rng.uniform(-1, 1, (6, hq, d)) * size
    x[1] *= 2.0 ** -3 if size < 1 else 2.0 ** -9
    x[2, :, 7] = size * (1 - 2.0 ** -24)
    q = torch.from_numpy(x).float().cuda()
    assert torch.isfinite(q).all()
    fresh, q64 = [3, 1, 2], q.double().cpu().numpy()
    o = ask("f32", c, q, fresh, lens, scale, shared)
    i = 0
    for b, m in enumerate(fresh):
        k, v, _ = c.tokens(b, lens[b])
        vis = np.arange(lens[b])[None, :] <= np.arange(m)[:, None] + (lens[b] - m)
        want = decoder.attend(q64[i:i + m], k, v, vis, scale)
        inside(o[i:i + m], want[0], tolerance("f32", *want, lens[b], d), "sequence %d" % b)
        i += m


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_step_longest_sequence(dtype):
    """A sequence of all the tokens that a page table may stand for, with pages for its first and its last ones only."""
    torch = torch_()
    rng = np.random.default_rng(4)
    d, page, held = 32, 512, 0x7fff0000
    width = held // page
    print("case: longest sequence", dtype, flush=True)
    c = Paged(rng, [2 * page], 1, d, page, spare=1)
    c.oracle.data[..., 32 * d:] = 125
    c.device.copy_(torch.from_numpy(c.oracle.data))
    k, v, _ = c.tokens(0, 2 * page)
    first, last = c.rows[0]
    c.table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    c.table[0, 0], c.table[0, width - 1] = int(first), int(last)
    c.desc = binding.kv4_desc(1, d, page, c.pages, 1, width)
    q, q64 = rows_of(rng, 2, 3, d, dtype, "plain")
    o = ask(dtype, c, q, [2], [held], 0.125, True)
    vis = np.ones((2, 2 * page), dtype=bool)
    vis[0, -1] = False
    want = decoder.attend(q64, k, v, vis, 0.125)
    inside(o, want[0], tolerance(dtype, *want, 2 * page, d), "the longest")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("announced", [0, 7, 0x7fff0000])
def test_prompt_keys_are_seen_whatever_was_announced(dtype, announced):
    """The announced longest of the keys orders the work and no more."""
    torch = torch_()
    rng = np.random.default_rng(12)
    qs, ks, d = [40, 300, 1], [90, 300, 700], 64
    print("case: announced keys", dtype, announced, flush=True)
    (q, q64), (k, k64), (v, v64) = (rows_of(rng, rows, 2, d, dtype, "plain") for rows in (sum(qs), sum(ks), sum(ks)))
    raw, o = empty(sum(qs), 2, d, dtype)
    cq, ck = sums(qs), sums(ks)
    desc = binding.prompt_desc(binding.DTYPES[dtype], 3, 2, 2, d, sum(qs), sum(ks), max(qs), announced, 0.125, 1, two(q), two(k), two(v), two(o))
    binding.ogc_prompt_run(desc, q.data_ptr(), k.data_ptr(), v.data_ptr(), cq.data_ptr(), ck.data_ptr(), o.data_ptr(), stream())
    torch.cuda.synchronize()
    i = j = 0
    for a, b in zip(qs, ks):
        vis = np.arange(b)[None, :] <= np.arange(a)[:, None] + (b - a)
        want = decoder.attend(q64[i:i + a], k64[j:j + b], v64[j:j + b], vis, 0.125)
        inside(o[i:i + a], want[0], tolerance(dtype, *want, b, d), "sequence of %d and %d" % (a, b))
        i, j = i + a, j + b
    assert untouched(raw)


@pytest.mark.parametrize("body,dtype", [("stream", "bf16"), ("few", "bf16"), ("split", "f32"), ("staged", "bf16"), ("staged", "f32")])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("what", ["lowest", "-inf"])
def test_prompt_first_scores_beyond_the_range(body, dtype, d, what):
    """The first seventy keys' scores are minus infinity for every row that sees them (padding of the lowest value, say), all others' far below zero: the rows that
    see others have the weighted mean of those."""
    torch = torch_()
    bad = float("-inf") if what == "-inf" else float(torch.finfo(dt(dtype)).min)
    qs, ks, far = [100, 40], [170, 40], -300.0

    def spoil(q, k, v):
        q[:] = q.abs().clamp(0.5, 2.0)
        k[:] = (k.double() * 0.01 + far / (d ** 0.5 * 1.1)).to(k.dtype)
        k[:70] = bad

    # (the common check says nothing here: a score that is off by a part of the largest one may be any)
    seen = {}
    kernel = {"stream": streams(d), "staged": "ogc_prompt_kernel<%d, %d>" % (binding.DTYPES[dtype], d // 32)}.get(body, "ogc_prompt_%s_kernel<%d>" % (body, d // 32))
    kw = dict(wide=(WIDE[dtype], 0), copies=1) if body == "staged" else {}
    o = prompts(kernel, dtype, qs, ks, 2, 1, d, d, spoil=lambda q, k, v: (spoil(q, k, v), seen.update(q=q.clone(), k=k.clone(), v=v.clone())), **kw)
    q, k, v = (seen[x].double().cpu().numpy() for x in "qkv")
    scale = float(np.float32(d ** -0.5))
    vis = np.arange(100)[None, :] <= np.arange(100)[:, None]
    want = decoder.attend(q[:100], k[70:170], v[70:170], vis, scale)
    assert np.abs(want[2]).min() > 100
    inside(o[:100], want[0], tolerance(dtype, *want, 170, d), "the rows' own keys")
