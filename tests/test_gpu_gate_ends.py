"""Gated rows (include/ogc_mx.h) whose gates are next to the ends of fp32, against oracle/mx.py in 64 bits: exp(-|a|) and a themselves below the normal numbers, where b may be as large as they are small.

The fp32 value is off by R = 2^-21 |y| (exponential and its argument 2^-22, sum, quotient and products 2^-22 more), and by half of the smallest fp32 number; a value read back from its format
by half a step more, 2^-4 |y| and 2^-10 of the scale (MX8), 1/4 |y| and 1/4 of the scale (MX4)."""
import numpy as np
import pytest

from oracle import mx
from paper_2301_01333_amd import binding

pytestmark = pytest.mark.gpu


def check(dtype, fmt, a, b):
    import torch

    n, c = a.shape
    print("case: gate", dtype, fmt, a.shape, a.min(), a.max(), flush=True)
    x = torch.from_numpy(np.concatenate([a, b], 1)).to({"bf16": torch.bfloat16, "f32": torch.float32}[dtype]).cuda()
    a, b = x[:, :c].double().cpu().numpy(), x[:, c:].double().cpu().numpy()
    kind = {"mx4": binding.OGC_MX4, "mx8": binding.OGC_MX8}[fmt]
    codes, scales = (torch.zeros(v, dtype=torch.uint8, device="cuda") for v in binding.ogc_mx_bytes(kind, n, c))
    binding.ogc_mx_write(binding.mx_rows(binding.DTYPES[dtype], kind, n, c, binding.OGC_GATE_SILU, x.stride(0)), x.data_ptr(), codes.data_ptr(), scales.data_ptr(),
                         int(torch.cuda.current_stream().cuda_stream))
    code, e = mx.codes_of(codes.cpu().numpy(), scales.cpu().numpy(), n, c, kind)
    want, got, scale = mx.gated(a, b), mx.values(code, e[:, ::32], kind)[:, :c], np.exp2(e.astype(float) - 127.0)[:, :c]
    assert (e < 255).all()
    R = 2.0 ** -21 * np.abs(want) + 2.0 ** -150
    top = lambda v: np.repeat(v.reshape(n, -1, 32).max(-1), 32, 1)  # noqa: E731 (of a group)
    low, high = (np.repeat(mx.quantize(top(v), kind)[1], 32, 1) for v in (np.maximum(np.abs(want) - R, 0), np.abs(want) + R))
    bad = ~((e[:, :c] == low) | (e[:, :c] == high))
    assert not bad.any(), (a[bad][::32][:4], b[bad][::32][:4], e[:, :c][bad][::32][:4], low[bad][::32][:4], want[bad][::32][:4])
    tol = (np.abs(want) / 16 + scale * 2.0 ** -10 if fmt == "mx8" else np.abs(want) / 4 + scale / 4) + 1.1 * R
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (a[bad][:4], b[bad][:4], got[bad][:4], want[bad][:4])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["mx4", "mx8"])
def test_gates_whose_exponential_is_below_the_normal_numbers(dtype, fmt):
    """Groups of gates that are all next to each other, with b of 1 and up to what keeps the product a number."""
    rng = np.random.default_rng(1)
    centre = np.array([-79.9, -80.1, -86.0, -87.3, -87.4, -88.0, -88.7, -90.0, -95.0, -103.0, -103.9, -104.1, -110.0, -127.9, -128.1, -150.0, -175.0, -190.0, -198.0, -230.0, -255.9, -256.1, -300.0, -511.0, -513.0, -1e4,
                       -1e30, -3e38])
    a = np.repeat(centre, 32).reshape(-1, 32) * (1 + 1e-4 * rng.random((len(centre), 32)))
    for size in (1.0, 2.0 ** 20, 2.0 ** 127, 2.0 ** -30):
        check(dtype, fmt, a, (1 + rng.random(a.shape)) * 0.75 * size * rng.choice([-1, 1], a.shape))
    # one far gate among ordinary ones
    ordinary = rng.normal(size=(40, 256))
    ordinary[::3, ::11] = -88.0 - 20 * rng.random(ordinary[::3, ::11].shape)
    check(dtype, fmt, ordinary, rng.normal(size=ordinary.shape))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["mx4", "mx8"])
def test_the_smallest_gates(dtype, fmt):
    """a below and next to the normal numbers: half of a * b, as large as b makes it."""
    rng = np.random.default_rng(2)
    step = 2.0 ** (-133 if dtype == "bf16" else -149)
    a = np.concatenate([step * rng.integers(-9, 10, (8, 64)), 2.0 ** -126 * rng.uniform(-4, 4, (8, 64)), np.zeros((1, 64))])
    for size in (1.0, 2.0 ** 60, 2.0 ** 126):
        check(dtype, fmt, a, (1 + rng.random(a.shape)) * size)
