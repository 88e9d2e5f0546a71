"""The choice of a token (include/ogc_sample.h) through the C ABI against oracle/mx.py.

Tokens are equal, wherever no decision was closer than vocab * 2^-42 of the sum it is compared with: weights are off by 2^-43 of the largest each when they are rounded, the
oracle's exponential and the kernel's by 2^-45 more, and no more than all of them add up.  Log-probabilities are rounded to fp32 once: 2^-24 of their value, and 2^-30 for the sum."""
import numpy as np
import pytest

from oracle import mx
from paper_2301_01333_amd import binding

pytestmark = pytest.mark.gpu


def torch_():
    import torch

    return torch


def stream():
    return int(torch_().cuda.current_stream().cuda_stream)


def run(logits, dtype, stride=None, offset=0, logs=True, **limits):
    """Tokens and log-probabilities of rows, and the logits in 64 bits; limits: arrays or None."""
    torch = torch_()
    rows, vocab = logits.shape
    t = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    stride = stride or vocab
    flat = torch.full((rows * stride + offset,), float("inf"), dtype=t, device="cuda")  # (what is between the rows would win)
    x = flat[offset:].reshape(rows, stride)[:, :vocab]
    x.copy_(torch.from_numpy(np.asarray(logits)).to(t))
    dev = {k: None if v is None else torch.tensor(np.asarray(v), dtype=torch.int32 if k == "top_k" else torch.float32, device="cuda") for k, v in limits.items()}
    p = lambda k: dev[k].data_ptr() if dev.get(k) is not None else 0  # noqa: E731
    token = torch.full((rows + 1,), -77, dtype=torch.int32, device="cuda")
    logp = torch.full((rows + 1,), -77.0, dtype=torch.float32, device="cuda")
    desc = binding.sample_desc(binding.DTYPES[dtype], rows, vocab, stride)
    space = torch.full((binding.ogc_sample_workspace_bytes(desc) + 16,), 0xEE, dtype=torch.uint8, device="cuda")
    binding.ogc_sample_run(desc, x.data_ptr(), p("temperature"), p("top_k"), p("top_p"), p("min_p"), p("uniform"), token.data_ptr(), logp.data_ptr() if logs else 0,
                           space.data_ptr(), stream())
    assert int(token[rows]) == -77 and float(logp[rows]) == -77.0 and (space[-16:] == 0xEE).all()
    return token[:rows].cpu().numpy(), logp[:rows].double().cpu().numpy(), x.double().cpu().numpy()


def check(logits, dtype, what, skipped=0.02, slack=0.0, **limits):
    """`skipped`: share of rows whose decisions may be too close to be sure of; `slack`: what the log of a sum of weights may be off by beyond its rounding."""
    rows = logits.shape[0]
    more = {k: limits.pop(k) for k in ("stride", "offset") if k in limits}
    print("case: sample", what, dtype, logits.shape, sorted(limits), more, flush=True)
    limits = {k: None if v is None else np.broadcast_to(np.asarray(v, dtype=np.int32 if k == "top_k" else np.float32), (rows,)) for k, v in limits.items()}
    token, logp, x = run(logits, dtype, **more, **limits)
    unsure = 0
    for r in range(rows):
        kw = {k: v[r].item() for k, v in limits.items() if v is not None}
        want, wantlog, margin = mx.sample(x[r], **kw)
        if margin < x.shape[1] * 2.0 ** -42:
            unsure += 1
            continue
        assert token[r] == want, (what, r, kw, int(token[r]), want, margin)
        assert logp[r] == wantlog or abs(logp[r] - wantlog) <= 2.0 ** -24 * abs(wantlog) + 2.0 ** -30 + slack, (what, r, logp[r], wantlog)
    assert unsure <= skipped * rows + 1
    return token


def some(rng, rows, vocab, sigma=3.0):
    x = rng.normal(size=(rows, vocab)) * sigma
    x[rng.random((rows, vocab)) < 0.03] = -np.inf
    return x


LIMITS = [dict(), dict(top_k=1), dict(top_k=40), dict(top_p=0.9), dict(top_p=0.3), dict(min_p=0.05), dict(top_k=50, top_p=0.95, min_p=0.02), dict(temperature=0.0),
          dict(temperature=0.3), dict(temperature=5.0, top_p=0.99), dict(top_k=100000), dict(top_k=-3, top_p=1.5, min_p=-1.0), dict(top_p=0.0), dict(min_p=1.0), dict(min_p=3.0)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [1, 2, 63, 64, 65, 500, 1000, 1025, 4099])
@pytest.mark.parametrize("i", range(len(LIMITS)))
def test_limits(dtype, vocab, i):
    rng = np.random.default_rng(vocab * 100 + i)
    rows = 24
    check(some(rng, rows, vocab), dtype, "limits", uniform=rng.random(rows), **LIMITS[i])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [32000, 50001, 131072])
def test_large_vocabularies(dtype, vocab):
    rng = np.random.default_rng(vocab)
    for kw in LIMITS[:9]:
        check(some(rng, 3, vocab), dtype, "large", skipped=0.4, uniform=rng.random(3), **kw)
    x = some(rng, 3, vocab)
    x[:, rng.integers(0, vocab, 5)] += 12.0
    for kw in LIMITS[:9]:
        check(x, dtype, "peaked", skipped=0.4, uniform=rng.random(3), **kw)


@pytest.mark.parametrize("rows", [1, 2, 7, 64, 200])
def test_rows_with_limits_of_their_own(rows):
    rng = np.random.default_rng(rows)
    x = some(rng, rows, 3001)
    check(x, "f32", "own limits", uniform=rng.random(rows), temperature=rng.choice([0.0, 0.5, 1.0, 2.0], rows), top_k=rng.choice([0, 1, 3, 50, 1000, 5000], rows),
          top_p=rng.choice([0.1, 0.5, 0.9, 0.999, 1.0], rows), min_p=rng.choice([0.0, 0.0, 0.01, 0.3], rows))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_equal_logits_are_kept_from_the_lowest_index_on(dtype):
    vocab = 5000
    x = np.zeros((12, vocab))
    x[1::3] = -3.0
    x[1::3, ::7] = 1.0
    x[2::3, 100:4000] = 2.0
    u = np.linspace(0, 0.9999, 12)
    for kw in (dict(), dict(top_k=3), dict(top_k=900), dict(top_k=4999), dict(top_p=0.5), dict(top_p=0.0001), dict(top_k=2000, top_p=0.77), dict(min_p=0.9), dict(temperature=0.0)):
        check(x, dtype, "equal", uniform=u, skipped=0.5, **kw)
    zeros = np.where(np.arange(vocab) % 2, 0.0, -0.0)[None, :].repeat(4, 0)
    token = check(zeros, dtype, "signed zeros", uniform=[0.0, 0.26, 0.51, 0.99], top_k=100)
    assert token.max() < 100 and (np.diff(token) > 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_without_choice(dtype):
    x = np.full((8, 300), -np.inf)
    x[1, 77] = -5.0
    x[2] = np.nan
    x[3, 5], x[3, 6] = np.nan, -1e30
    x[4, 200], x[4, 210] = np.inf, np.inf
    x[5] = np.inf
    x[6, 299], x[6, 0] = 3e38, -3e38
    x[7] = 1.0
    for kw in (dict(), dict(top_k=2), dict(top_p=0.5), dict(min_p=0.5), dict(temperature=0.0), dict(temperature=float("nan")), dict(temperature=float("inf")), dict(temperature=1e-40),
               dict(top_p=float("nan"), min_p=float("nan"))):
        for u in (0.0, 0.7):
            token = check(x, dtype, "no choice %s" % kw, uniform=u, skipped=1.0, **kw)
            assert token[0] == -1 and token[1] == 77 and token[2] == -1 and token[3] == 6 and token[4] in (200, 210)


def test_uniforms_at_the_ends():
    x = np.log(np.array([[0.1, 0.4, 0.3, 0.2, 1e-30]])).repeat(6, 0)
    u = [0.0, -1.0, float("nan"), 1.0, 7.0, np.nextafter(np.float32(1), np.float32(0))]
    token, _, _ = run(x, "f32", uniform=u, temperature=None)
    assert token.tolist() == [0, 0, 0, 3, 3, 3]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_and_offsets(dtype):
    rng = np.random.default_rng(2)
    for vocab, stride, offset in ((1000, 1000, 1), (1001, 1003, 0), (1024, 1032, 3), (70, 71, 5)):
        check(some(rng, 5, vocab), dtype, "strides", stride=stride, offset=offset, uniform=rng.random(5), top_k=20, top_p=0.8)
    x = some(rng, 5, 100)
    a, _, _ = run(x, dtype, uniform=np.full(5, 0.4), logs=False)
    b, _, _ = run(x, dtype, uniform=np.full(5, 0.4))
    assert np.array_equal(a, b)


def test_rows_beyond_4_gib():
    torch = torch_()
    rng = np.random.default_rng(8)
    rows, vocab, stride = 3, 5000, (1 << 30) + 1
    flat = torch.empty((rows - 1) * stride + vocab, device="cuda")
    x = flat.as_strided((rows, vocab), (stride, 1))
    x.copy_(torch.from_numpy(some(rng, rows, vocab)))
    near = x.contiguous()
    u, k, share = torch.tensor([0.1, 0.5, 0.9], device="cuda"), torch.tensor([0, 30, 0], dtype=torch.int32, device="cuda"), torch.tensor([1.0, 0.9, 0.7], device="cuda")
    tokens = []
    for v, s in ((x, stride), (near, vocab)):
        desc = binding.sample_desc(0, rows, vocab, s)
        space, token = torch.empty(binding.ogc_sample_workspace_bytes(desc), dtype=torch.uint8, device="cuda"), torch.full((rows,), -7, dtype=torch.int32, device="cuda")
        binding.ogc_sample_run(desc, v.data_ptr(), 0, k.data_ptr(), share.data_ptr(), 0, u.data_ptr(), token.data_ptr(), 0, space.data_ptr(), stream())
        tokens.append(token.tolist())
    assert tokens[0] == tokens[1]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sigma,temperature", [(0.02, 1.0), (1.0, 0.05), (2.0, 1.5), (40.0, 1.0), (300.0, 30.0), (1e30, 1.0), (1e-30, 1e-28)])
def test_spreads(dtype, sigma, temperature):
    """Flat rows, whose limits have thousands of tokens before them, and steep ones; logits and temperatures of all sizes."""
    rng = np.random.default_rng(6)
    x = some(rng, 4, 20011, sigma)
    u = rng.random(4)
    for kw in (dict(top_p=0.97), dict(top_p=0.4), dict(min_p=0.3), dict(min_p=1e-6), dict(top_p=0.9, min_p=0.01), dict(top_p=0.2, min_p=0.001), dict(top_k=300), dict(top_k=1024, top_p=0.9),
               dict(top_k=1025, top_p=0.9, min_p=0.02), dict(top_k=19000), dict()):
        check(x, dtype, "spread %g %g %s" % (sigma, temperature, kw), skipped=0.5, temperature=temperature, uniform=u, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_limits_next_to_zero(dtype):
    """The bins' limits at logits of 0, -0 and the smallest numbers, where many tokens are."""
    rng = np.random.default_rng(8)
    x = rng.choice([0.0, -0.0, 1e-40, -1e-40, 1e-3, -1e-3, 0.5, -0.5, -0.03125, 0.03125], size=(6, 3000))
    x[:, 7] = [0.0, 0.25, 1.0, 0.03125, 2.0, 0.5]
    u = rng.random(6)
    for kw in (dict(top_p=0.5), dict(top_p=0.9), dict(min_p=0.96), dict(min_p=0.5), dict(top_p=0.7, min_p=0.9), dict(top_k=700), dict()):
        check(x, dtype, "zeros %s" % kw, skipped=0.5, uniform=u, **kw)
        check(x, dtype, "zeros %s" % kw, skipped=0.5, uniform=u, temperature=0.031, **kw)


@pytest.mark.parametrize("rows,vocab", [(1, 2048), (1, 2049), (3, 8193), (64, 128000), (1, 1 << 20), (2, 300001), (300, 5000)])
def test_parts(rows, vocab):
    """Parts of all sizes, one and many of them, with the chosen token in each."""
    rng = np.random.default_rng(vocab)
    x = some(rng, rows, vocab, 2.0)
    if rows > 8:
        x[8:] = x[rng.integers(0, 8, rows - 8)]
    few = np.arange(rows) if rows <= 8 else np.concatenate([np.arange(8), rng.integers(8, rows, 4)])
    for kw in (dict(), dict(top_p=0.95), dict(min_p=0.02), dict(top_k=77)):
        u = rng.random(rows).astype(np.float32)
        token, logp, x64 = run(x, "f32", uniform=u, **{k: np.full(rows, v) for k, v in kw.items()})
        for r in few:
            want, wantlog, margin = mx.sample(x64[r], uniform=u[r].item(), **{k: np.float32(v).item() if k != "top_k" else v for k, v in kw.items()})
            if margin >= vocab * 2.0 ** -42:
                assert token[r] == want and abs(logp[r] - wantlog) <= 2.0 ** -24 * abs(wantlog) + 2.0 ** -30, (kw, r, token[r], want)


def test_shares_of_many_draws():
    """Twenty thousand rows of the same logits: every kept token as often as its weight says, within five standard deviations."""
    rng = np.random.default_rng(11)
    n, x = 20000, np.array([0.3, -1.0, 2.0, 1.5, -9.0, 1.9, 0.0])
    token, logp, _ = run(x[None, :].repeat(n, 0), "f32", uniform=rng.random(n), top_k=np.full(n, 5))
    w = np.exp(x - x.max())
    w[[1, 4]] = 0.0
    w /= w.sum()
    share = np.bincount(token, minlength=7) / n
    assert (np.abs(share - w) <= 5 * np.sqrt(w * (1 - w) / n)).all()
    assert np.allclose(np.exp(logp), w[token], rtol=1e-5)


def test_in_a_graph():
    torch = torch_()
    rng = np.random.default_rng(3)
    rows, vocab = 5, 40000
    x = torch.from_numpy(rng.normal(size=(rows, vocab)) * 3).float().cuda()
    other = torch.from_numpy(rng.normal(size=(rows, vocab)) * 3).float().cuda()
    u, p, k = torch.rand(rows, device="cuda"), torch.full((rows,), 0.9, device="cuda"), torch.full((rows,), 300, dtype=torch.int32, device="cuda")
    desc = binding.sample_desc(0, rows, vocab, vocab)
    spaces = [torch.full((binding.ogc_sample_workspace_bytes(desc) + 16,), 0xEE, dtype=torch.uint8, device="cuda") for _ in range(2)]
    token, eager = (torch.zeros(rows, dtype=torch.int32, device="cuda") for _ in range(2))
    call = lambda out, space: binding.ogc_sample_run(desc, x.data_ptr(), 0, k.data_ptr(), p.data_ptr(), 0, u.data_ptr(), out.data_ptr(), 0, space.data_ptr(), stream())  # noqa: E731
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        call(token, spaces[0])
    for i in range(5):
        if i == 2:
            x.copy_(other)
        u.copy_(torch.rand(rows, device="cuda"))
        token.fill_(-5)
        g.replay()
        call(eager, spaces[1])
        torch.cuda.synchronize()
        assert torch.equal(token, eager) and (token >= 0).all()


@pytest.mark.parametrize("seed", range(6))
def test_limits_of_all_kinds_together(seed):
    """Rows of every kind with limits of their own: the weights are multiples of 2^-42 of a part's largest here and of a row's in the oracle, half of one off each."""
    rng = np.random.default_rng(seed)
    for i in range(20):
        rows, vocab = int(rng.integers(1, 9)), int(np.exp(rng.uniform(0, np.log(200000))))
        sigma = float(np.exp(rng.uniform(-3, 4)))
        x = rng.normal(size=(rows, vocab)) * sigma
        if i % 5 == 1:
            x = np.round(x * 2) / 2  # many equal ones
        elif i % 5 == 2:
            x[:, rng.integers(0, vocab, 3)] += 20
        elif i % 5 == 3:
            x = 1e3 * rng.normal() - rng.exponential(sigma, (rows, vocab)) ** 2
        elif i % 5 == 4:
            x[rng.random((rows, vocab)) < 0.9] = -np.inf
        if i % 7 == 0:
            x[rng.integers(0, rows), rng.integers(0, vocab)] = rng.choice([np.inf, np.nan])
        limits = dict(uniform=rng.random(rows), temperature=rng.choice([0.0, 1e-3, 0.1, 0.7, 1.0, 1.5, 10.0, 1e3], rows))
        if rng.random() < 0.6:
            limits["top_k"] = rng.choice([0, 1, 2, 40, 100, 500, 1000, 1024, 1025, 3000], rows)
        if rng.random() < 0.6:
            limits["top_p"] = rng.choice([1.0, 0.9, 0.5, 0.99, 0.05, 0.9999], rows)
        if rng.random() < 0.4:
            limits["min_p"] = rng.choice([0.0, 0.01, 0.1, 0.5, 1e-4, 1e-9], rows)
        dtype = str(rng.choice(["bf16", "f32"]))
        check(x, dtype, "together %d" % i, skipped=1.0, slack=vocab * 2.0 ** -42, stride=vocab + int(rng.integers(0, 9)), offset=int(rng.integers(0, 8)), **limits)
