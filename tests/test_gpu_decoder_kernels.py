"""Every kernel of the decoder's attention block on the inputs where it can go wrong: each call says which kernel it is for, so that a rule
that sends it elsewhere fails here.  (The calls of test_gpu_decoder.py are small: in bf16 they have few tiles, and over the cache hardly one
is shared by several workgroups.)  Oracle and tolerances: test_gpu_decoder.py."""
import numpy as np
import pytest

from oracle import decoder
from paper_2301_01333_amd import binding
from test_gpu_decoder import Paged, dt, empty, inside, ints, rows_of, stream, sums, tolerance, torch_, two, untouched

pytestmark = pytest.mark.gpu


# ---- prompts ----------------------------------------------------------------------------------------------------------------
def spread(x, stride):
    """x [rows, heads, d] with that many elements from row to row."""
    torch = torch_()
    flat = torch.empty(max(len(x) - 1, 0) * stride + x.shape[1] * x.shape[2], dtype=x.dtype, device="cuda")
    v = flat.as_strided(x.shape, (stride, x.shape[2], 1))
    v.copy_(x)
    return v


def prompts(kernel, dtype, qs, ks, hq, hk, d, seed, order="plain", causal=1, spoil=None, loud=1.0, max_q=None, copies=None, wide=(), finite=None):
    """hk key heads and their query heads `copies` times over (None: as often as it takes to come to that kernel): the first ones are held to the
    oracle, the others to their bytes.  wide: strides from row to row of keys and values, in elements."""
    torch = torch_()
    print("case: prompts", kernel, dtype, qs, ks, hq, hk, d, order, causal, flush=True)
    rng = np.random.default_rng(7000 + seed)
    n, m, scale = sum(qs), sum(ks), float(np.float32(d ** -0.5))
    q, k, v = (rows_of(rng, rows, heads, d, dtype, "plain", by)[0] for rows, heads, by in ((n, hq, loud), (m, hk, 1.0), (m, hk, 1.0)))
    if spoil:
        spoil(q, k, v)
    q64, k64, v64 = (x.double().cpu().numpy() for x in (q, k, v))
    most = max(qs) if max_q is None else max_q
    for times in ([copies] if copies else [2 ** i for i in range(10)]):
        shapes = [(rows, heads * times, d) for rows, heads in ((n, hq), (m, hk), (m, hk))]
        strides = [(d, rows * d) if order == "heads" else (heads * d, d) for rows, heads, _ in shapes]
        strides = [strides[0]] + [(w or s[0], s[1]) for w, s in zip(wide or (0, 0), strides[1:])]
        desc = binding.prompt_desc(binding.DTYPES[dtype], len(qs), hq * times, hk * times, d, n, m, most, max(ks), scale, causal, *strides, (hq * times * d, d))
        if binding.ogc_prompt_kernel_name(desc) == kernel:
            break
    assert binding.ogc_prompt_kernel_name(desc) == kernel
    q, k, v = (x.repeat(1, times, 1) for x in (q, k, v))
    if order == "heads":
        q, k, v = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v))
    if wide:
        k, v = (spread(x, w) if w else x for x, w in zip((k, v), wide))
    raw, o = empty(n, hq * times, d, dtype)
    cq, ck = sums(qs), sums(ks)
    binding.ogc_prompt_run(desc, q.data_ptr(), k.data_ptr(), v.data_ptr(), cq.data_ptr(), ck.data_ptr(), o.data_ptr(), stream())
    i = j = 0
    for s, (a, b) in enumerate(zip(qs, ks)):
        vis = np.arange(b)[None, :] <= np.arange(a)[:, None] + (b - a) if causal else np.ones((a, b), dtype=bool)
        with np.errstate(invalid="ignore"):
            want = decoder.attend(q64[i:i + a], k64[j:j + b], v64[j:j + b], vis, scale)
            tol = tolerance(dtype, *want, b, d)
        look = min(a, most, finite[s] if finite else a)
        inside(o[i:i + look, :hq], want[0][:look], tol[:look], "sequence of %d and %d" % (a, b))
        if a > most:  # rows beyond the announced longest are left as they are
            assert bool((o[i + most:i + a].contiguous().view(torch.uint8) == 0xCD).all())
        i, j = i + a, j + b
    assert untouched(raw)
    for c in range(1, times):
        assert torch.equal(o[:, :hq].contiguous().view(torch.uint8), o[:, c * hq:(c + 1) * hq].contiguous().view(torch.uint8)), "copy %d" % c
    return o[:, :hq]


def streams(d):
    return "ogc_prompt_stream_kernel<%d>" % (d // 32)


@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("hq,hk", [(2, 2), (6, 2), (8, 1), (7, 1)])
def test_stream_heads_and_lengths(d, hq, hk):
    prompts(streams(d), "bf16", [70, 1, 40], [70, 1, 40], hq, hk, d, hq + d)
    lens = [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200]
    prompts(streams(d), "bf16", lens, lens, hq, hk, d, hq + d)


@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("causal", [1, 0])
@pytest.mark.parametrize("qs,ks", [([5, 0, 3], [50, 4, 0]), ([9, 70, 1], [3, 69, 300]), ([33, 64], [131, 257]), ([40, 2, 90], [7, 1, 90]), ([333, 130, 257], [333, 200, 257])])
def test_stream_earlier_keys_and_rows_that_see_nothing(d, causal, qs, ks):
    prompts(streams(d), "bf16", qs, ks, 4, 2, d, sum(qs), causal=causal)


@pytest.mark.parametrize("d", [32, 64, 96, 128])
def test_stream_one_sequence(d):
    """A single sequence is handed out without sorting."""
    prompts(streams(d), "bf16", [300], [420], 3, 1, d, 11)


@pytest.mark.parametrize("d", [32, 64, 96, 128])
def test_stream_orders_and_rows_left_out(d):
    prompts(streams(d), "bf16", [70, 20], [90, 20], 4, 2, d, 3, "heads")
    prompts(streams(d), "bf16", [90, 10], [90, 10], 4, 2, d, 3, max_q=64)


def hidden(bad):
    def spoil(q, k, v):
        k[60:70], v[60:70] = bad, bad
        v[100, :, 5] = bad          # the second sequence's own last token, one channel
        k[100 + 30], v[100 + 45] = bad, bad

    return spoil


def late(q, k, v):
    k *= torch_().linspace(0.1, 3.0, len(k), device="cuda")[:, None, None].to(k.dtype)


NO_NUMBERS = {"nan": float("nan"), "inf": float("inf"), "-inf": float("-inf")}


def no_numbers(kernel, dtype, d, what, **kw):
    """Keys and values of later tokens hold no numbers: rows before them are what they are without them."""
    torch = torch_()
    bad = NO_NUMBERS.get(what, float(torch.finfo(dt(dtype)).min))
    o = prompts(kernel, dtype, [70, 31, 60], [70, 31, 60], 4, 2, d, 5, spoil=hidden(bad), finite=[60, 30, 29] if what == "lowest" else None, **kw).cpu()
    assert torch.isfinite(o[:60]).all() and torch.isfinite(o[70:100]).all()
    if what != "lowest":
        assert not torch.isfinite(o[100, :, 5]).any() and torch.isfinite(o[100, :, :5]).all()


@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("what", ["nan", "inf", "-inf", "lowest"])
def test_stream_no_numbers_where_a_row_does_not_see_them(d, what):
    no_numbers(streams(d), "bf16", d, what)


@pytest.mark.parametrize("d", [32, 64, 96, 128])
def test_stream_large_scores(d):
    prompts(streams(d), "bf16", [150, 40], [200, 40], 4, 2, d, 8, spoil=late, loud=20.0)


WIDE = {"bf16": (1 << 25) + 64, "f32": (1 << 22) + 32}  # elements from row to row that the other bodies' offsets do not hold


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
def test_rows_far_apart(dtype, d):
    """Token strides of 64 MiB (bf16) and 16 MiB and more: the staged body as a kernel of its own."""
    kernel = "ogc_prompt_kernel<%d, %d>" % (binding.DTYPES[dtype], d // 32)
    for wide in ((WIDE[dtype], 0), (0, WIDE[dtype])):
        prompts(kernel, dtype, [33, 7], [50, 20], 6, 2, d, d, wide=wide, copies=1)
    prompts(kernel, dtype, [20, 3, 2], [40, 0, 1], 4, 2, d, d, wide=(WIDE[dtype], 0), copies=1, causal=0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,what", [(32, "nan"), (64, "inf"), (96, "-inf"), (128, "lowest")])
def test_rows_far_apart_no_numbers_and_large_scores(dtype, d, what):
    kernel = "ogc_prompt_kernel<%d, %d>" % (binding.DTYPES[dtype], d // 32)
    no_numbers(kernel, dtype, d, what, wide=(0, WIDE[dtype]), copies=1)
    prompts(kernel, dtype, [60, 40], [80, 40], 2, 1, d, 8, spoil=late, loud=20.0, wide=(WIDE[dtype], 0), copies=1)


# ---- attention over the cache -----------------------------------------------------------------------------------------------
def steps(dtype, fresh, lens, hq, hk, d, page, seed, shared, holes=(), spoil=None, loud=1.0):
    """shared: whether several workgroups have a sequence (a workspace is asked for).  The cache holds random codes with moderate scales."""
    torch = torch_()
    print("case: steps", dtype, fresh, lens, hq, hk, d, page, shared, flush=True)
    rng = np.random.default_rng(8000 + seed)
    c = Paged(rng, lens, hk, d, page, holes=holes)
    c.oracle.data[..., 32 * d:] = rng.integers(120, 127, c.oracle.data[..., 32 * d:].shape)
    if spoil:
        spoil(c)
    c.device.copy_(torch.from_numpy(c.oracle.data))
    n, most, scale = sum(fresh), max(lens), float(np.float32(d ** -0.5))
    q, q64 = rows_of(rng, n, hq, d, dtype, "slice", loud)
    raw, o = empty(n, hq, d, dtype)
    cu, ln = sums(fresh), ints(lens)
    desc = binding.kv4_attention_desc(binding.DTYPES[dtype], hq, n, max(fresh), most, scale, two(q), two(o))
    need = binding.ogc_kv4_attention_workspace_bytes(c.desc, desc)
    assert (need > 0) == shared
    ws = torch.full((max(16, need),), 0xFF, dtype=torch.uint8, device="cuda")
    binding.ogc_kv4_attention_run(c.desc, desc, q.data_ptr(), cu.data_ptr(), ln.data_ptr(), c.table.data_ptr(), c.device.data_ptr(), o.data_ptr(), ws.data_ptr(), stream())
    i = 0
    for b, m in enumerate(fresh):
        k, v, there = c.tokens(b, lens[b])
        vis = (np.arange(lens[b])[None, :] <= np.arange(m)[:, None] + (lens[b] - m)) & there[None, :]
        want = decoder.attend(q64[i:i + m], k, v, vis, scale)
        inside(o[i:i + m], want[0], tolerance(dtype, *want, lens[b], d), "sequence %d" % b)
        i += m
    assert untouched(raw)
    return o


LENS = [1500, 0, 700, 1, 33, 1290, 128]
HOLES = [(0, 2, -1), (0, 3, 1 << 29), (2, 10, -5), (5, 0, -1)]  # a whole split of the first sequence, ends of others


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
def test_shared_sequences(dtype, d):
    """Lengths all different, empty ones, one query each; then with pages missing."""
    one = [1] * len(LENS)
    steps(dtype, one, LENS, 4, 2, d, 64, d, True)
    steps(dtype, one, LENS, 4, 2, d, 64, d, True, holes=HOLES, loud=20.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("fresh,hq", [([3, 0, 1, 2, 40, 5, 1], 2), ([2, 1, 1, 1, 2, 7, 3], 24)])
def test_shared_sequences_several_queries(dtype, d, fresh, hq):
    """More queries than tokens, and (bf16) columns for one tile of 16 and for two."""
    steps(dtype, fresh, LENS, hq, 2, d, 32, d + hq, True, holes=[(0, 5, -1)])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
def test_shared_sequences_no_numbers(dtype, d):
    """Byte 255 where a token is seen spoils what sees it, whichever split it is in."""
    torch = torch_()

    def spoil(c):
        at = lambda b, t: (c.rows[b][t // 64], t % 64 // 32, t % 32)  # noqa: E731
        page, block, t = at(0, 1499)
        c.oracle.data[page, 0, block, 32 * d + t] = 255      # the last key of the first sequence, head 0
        page, block, t = at(2, 300)
        c.oracle.data[page, 1, block, 33 * d + t] = 255      # a value's first 32 channels, head 1
        page, block, t = at(5, 1290)                         # behind the last token
        c.oracle.data[page, :, block, [32 * d + t, 33 * d + t]] = 255

    o = torch.isnan(steps(dtype, [2] + [1] * 6, LENS, 4, 2, d, 64, d, True, spoil=spoil)).cpu()
    assert not o[0].any() and o[1, :2].all() and not o[1, 2:].any()  # (the first query of two does not see the last token)
    assert o[3, 2:, :32].all() and o[3].sum() == 2 * 32
    assert not o[2].any() and not o[4:].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("hq", [16, 48])
def test_sequences_of_one_workgroup_of_four_wavefronts(dtype, d, hq):
    """Batches that fill the chip: a sequence is one workgroup's, of any length; one column tile and (bf16, several queries) two."""
    rng = np.random.default_rng(d)
    lens = rng.integers(1, 60, 48).tolist()
    lens[0], lens[7], lens[9] = 300, 0, 161
    fresh = [1] * 48 if hq == 16 else [1 + i % 7 for i in range(48)]
    steps(dtype, fresh, lens, hq, 16, d, 32, d + hq, False, holes=[(0, 3, -1), (9, 0, -1)])
