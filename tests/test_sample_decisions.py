"""How sure the oracle's choice of a token is (oracle/mx.py): its margin, by which tests leave out rows whose decisions are closer than the weights' own rounding, is no larger than what really
changes a row's token, and so large that hardly a row is left out; and on the GPU the choice in rows of every kind (include/ogc_sample.h), of which next to none may be left out.

Weights are multiples of 2^-42 of the largest; a log-probability is rounded to fp32, 2^-24 of its value, its sum of weights is off by vocab * 2^-42 at most, and 2^-30 stands for the rest."""
import numpy as np
import pytest

from oracle import mx


def kinds(seed, count):
    """Rows of every kind with limits of their own: (logits [rows, vocab], limits)."""
    rng = np.random.default_rng(seed)
    for i in range(count):
        rows, vocab = int(rng.integers(1, 9)), int(np.exp(rng.uniform(0, np.log(150000))))
        sigma = float(np.exp(rng.uniform(-3, 4)))
        x = rng.normal(size=(rows, vocab)) * sigma
        if i % 5 == 1:
            x[:, rng.integers(0, vocab, 3)] += 20
        elif i % 5 == 2:
            x = 1e3 * rng.normal() - rng.exponential(sigma, (rows, vocab)) ** 2
        elif i % 5 == 3:
            x[rng.random((rows, vocab)) < 0.9] = -np.inf
        if i % 7 == 0:
            x[rng.integers(0, rows), rng.integers(0, vocab)] = rng.choice([np.inf, np.nan])
        limits = dict(uniform=rng.random(rows), temperature=rng.choice([0.0, 0.1, 0.7, 1.0, 1.5, 10.0], rows))
        if i % 3:
            limits["top_k"] = rng.choice([0, 1, 2, 40, 100, 500, 1000, 1024, 1025, 3000], rows)
        if i % 2:
            limits["top_p"] = rng.choice([1.0, 0.9, 0.51, 0.99, 0.05, 0.9999], rows)
        if i % 4 == 1:
            limits["min_p"] = rng.choice([0.0, 0.01, 0.1, 0.5, 1e-4], rows)
        yield x.astype(np.float32).astype(float), {k: np.asarray(v, dtype=np.int32 if k == "top_k" else np.float32) for k, v in limits.items()}


def of_row(limits, r):
    return {k: v[r].item() for k, v in limits.items()}


def test_hand_cases():
    row = np.log(np.array([0.5, 0.3, 0.2]))
    for kw, margin in ((dict(uniform=0.4), 0.1), (dict(uniform=0.7), 0.1), (dict(uniform=0.4, top_p=0.6), 0.1), (dict(uniform=0.6, top_p=0.6), 0.025), (dict(uniform=0.1, min_p=0.35), 0.05),
                       (dict(uniform=0.1, top_k=1), np.inf), (dict(uniform=0.5), 0.0), (dict(uniform=0.2, top_p=0.8), 0.0)):
        assert mx.sample(row, **kw)[2] == pytest.approx(margin, abs=1e-6), kw


@pytest.mark.parametrize("seed", range(3))
def test_hardly_a_row_is_left_out_and_none_changes_within_its_margin(seed):
    rows = unsure = 0
    for x, limits in kinds(seed, 30):
        for r in range(len(x)):
            kw = of_row(limits, r)
            token, _, margin = mx.sample(x[r], **kw)
            rows += 1
            unsure += margin < x.shape[1] * 2.0 ** -42
            step = min(0.9 * margin, 0.1)
            for name in ("uniform", "top_p", "min_p"):
                if 0 < kw.get(name, 0.0) < 1 and kw["temperature"] > 0 and np.isfinite(margin):
                    for way in (-step, step):
                        other = dict(kw, **{name: kw[name] + way})
                        if 0 < other[name] < 1:
                            assert mx.sample(x[r], **other)[0] == token, (kw, name, margin)
    assert unsure <= 0.03 * rows


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(10, 16))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_every_kind(seed, dtype):
    import torch

    from paper_2301_01333_amd import binding

    t = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    checked = unsure = 0
    for x, limits in kinds(seed, 20):
        rows, vocab = x.shape
        print("case: kinds", seed, dtype, x.shape, sorted(limits), flush=True)
        logits = torch.from_numpy(x).to(t).cuda()
        dev = {k: torch.from_numpy(v).cuda() for k, v in limits.items()}
        p = lambda k: dev[k].data_ptr() if k in dev else 0  # noqa: E731
        desc = binding.sample_desc(binding.DTYPES[dtype], rows, vocab, vocab)
        space = torch.empty(binding.ogc_sample_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
        token, log = torch.full((rows,), -9, dtype=torch.int32, device="cuda"), torch.full((rows,), -9.0, device="cuda")
        binding.ogc_sample_run(desc, logits.data_ptr(), p("temperature"), p("top_k"), p("top_p"), p("min_p"), p("uniform"), token.data_ptr(), log.data_ptr(), space.data_ptr(),
                               int(torch.cuda.current_stream().cuda_stream))
        token, log, x = token.cpu().numpy(), log.double().cpu().numpy(), logits.double().cpu().numpy()
        for r in range(rows):
            want, wantlog, margin = mx.sample(x[r], **of_row(limits, r))
            if margin < vocab * 2.0 ** -42:
                unsure += 1
                continue
            checked += 1
            assert token[r] == want, (r, of_row(limits, r), token[r], want, margin)
            assert log[r] == wantlog or abs(log[r] - wantlog) <= 2.0 ** -24 * abs(wantlog) + 2.0 ** -30 + vocab * 2.0 ** -42, (r, log[r], wantlog)
    assert unsure <= 0.04 * checked + 1 and checked >= 60
