"""The norm (include/ogc_mx.h) of rows from the smallest to the largest numbers, with an eps of 0 and others, and its accuracy whatever a row's length, against oracle/mx.py in 64 bits.

The squares, their sum and the root are held in 64 bits: some c * 2^-53, nothing here.  The factor is rounded to fp32 (2^-24), a value's products with it and with the weight 2^-24 each: 3 * 2^-24 |y|, and
as much again of 2^-24 for the squares of these.  Then the type's own rounding, half a step, or that of a format: half a step, 2^-4 |y| and 2^-10 of the scale (MX8), 1/4 |y| and 1/4 of the scale (MX4)."""
import numpy as np
import pytest

from oracle import mx
from paper_2301_01333_amd import binding

pytestmark = pytest.mark.gpu
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
TINY = {"bf16": 2.0 ** -134, "f32": 2.0 ** -150}
OUTS = {"same": 0, "mx4": 1, "mx8": 2}


def norm(dtype, x, out, eps, weight, residual=None):
    """The norm of rows (of their sum) and that sum, in 64 bits; a matrix as its values with its scales."""
    import torch

    t = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    n, c = x.shape

    def rows(v):
        r = torch.full((n, mx.up(c, 8)), 55.0, dtype=t, device="cuda")
        if v is not None:
            r[:, :c] = torch.from_numpy(v).to(t)
        return r

    xd, y, w = rows(x), rows(None), torch.from_numpy(weight).float().cuda()
    rd, s = (None, xd) if residual is None else (rows(residual), rows(None))
    wide = xd.stride(0)
    desc = binding.norm_desc(binding.DTYPES[dtype], n, c, OUTS[out], eps, wide, wide if rd is not None else 0, wide if rd is not None else 0, wide if out == "same" else 0)
    codes, scales = (torch.full((max(b, 16),), 0xCD, dtype=torch.uint8, device="cuda") for b in binding.ogc_mx_bytes(binding.OGC_MX4 if out == "mx4" else binding.OGC_MX8, n, c))
    binding.ogc_norm_run(desc, xd.data_ptr(), 0 if rd is None else rd.data_ptr(), w.data_ptr(), 0 if rd is None else s.data_ptr(), y.data_ptr() if out == "same" else codes.data_ptr(),
                         0 if out == "same" else scales.data_ptr(), int(torch.cuda.current_stream().cuda_stream))
    s64 = s[:, :c].double().cpu().numpy()
    if out == "same":
        assert bool((y[:, c:] == 55.0).all())
        return s64, w.double().cpu().numpy(), y[:, :c].double().cpu().numpy(), None
    fmt = mx.MX4 if out == "mx4" else mx.MX8
    code, e = mx.codes_of(codes.cpu().numpy(), scales.cpu().numpy(), n, c, fmt)
    return s64, w.double().cpu().numpy(), mx.values(code, e[:, ::32], fmt)[:, :c], np.exp2(e.astype(float) - 127.0)[:, :c]


def check(dtype, x, out, eps, weight=None, residual=None):
    print("case: norm", dtype, x.shape, out, eps, residual is not None, flush=True)
    weight = np.ones(x.shape[1]) if weight is None else weight
    s, w, got, scale = norm(dtype, x, out, eps, weight, residual)
    with np.errstate(invalid="ignore"):
        want = mx.norm(s, w, eps)  # (a sum may be an infinity: NaN, and zeros beside it)
    if out != "same":  # a group that holds no number is none
        none = np.isnan(np.pad(want, ((0, 0), (0, -want.shape[1] % 32)))).reshape(len(want), -1, 32).any(-1)
        want = np.where(np.repeat(none, 32, axis=1)[:, :want.shape[1]], np.nan, want)
    R = 3.001 * 2.0 ** -24 * np.abs(want) + 2.0 ** -149  # (products below the normal numbers: half of the smallest one each)
    if out == "same":
        tol = HALF[dtype] * np.abs(want) + TINY[dtype] + R
    elif out == "mx8":
        tol = np.abs(want) / 16 + scale * 2.0 ** -10 + 1.1 * R
    else:
        tol = np.abs(want) / 4 + scale / 4 + 1.1 * R
    bad = ~((np.abs(got - want) <= tol) | (np.isnan(got) & np.isnan(want)))
    assert not bad.any(), (got[bad][:4], want[bad][:4])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("out", ["same", "mx4", "mx8"])
@pytest.mark.parametrize("n,c", [(13, 300), (13, 4096), (3, 20000), (8200, 250), (8200, 1000)])
def test_rows_of_all_sizes(dtype, out, n, c):
    """Rows of 2^-133 (bf16; fp32: 2^-140) to 2^125, whose squares are no fp32 numbers, one of ones and one of the largest and smallest side by side."""
    rng = np.random.default_rng(c)
    sizes = np.exp2(np.array([-133 if dtype == "bf16" else -140, -126, -110, -100, -76, -75, -64, -40, 0, 30, 61, 64, 80, 100, 120, 125], dtype=float))
    x = rng.normal(size=(n, c)).clip(-3.5, 3.5)
    x[:, 0] = 1.0  # (no row of zeros: nothing is their norm without eps)
    x *= sizes[np.arange(n) % len(sizes)][:, None]
    x[n // 2, ::2], x[n // 2, 1::2] = 3e38, 1e-38
    for eps in (0.0, 1e-6, 1e-30, 1e30):
        check(dtype, x, out, eps, 1 + 0.3 * rng.normal(size=c))
    check(dtype, x[:8], out, 0.0, residual=0.5 * x[:8])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v", [2.0 ** -133, 1e-30, 1e-23, 1e-22, 1e-21, 1.0, 2.0 ** 62, 1e30, 3e38])
def test_constant_rows_are_ones(dtype, v):
    for n, c in ((1, 8), (2, 9000)):
        x = np.full((n, c), v)
        x[:, ::3] *= -1
        for out in OUTS:
            check(dtype, x, out, 0.0)


@pytest.mark.parametrize("out", ["same", "mx8"])
@pytest.mark.parametrize("n,c", [(2, 66000), (2, 1 << 20), (40, 8192), (8193, 256)])
def test_the_factor_is_the_rounded_one_whatever_the_length(out, n, c):
    """A sum in fp32 would be off by 2^-24 for each addition.  Of values of one sign and a few sizes, so that errors do not even out."""
    rng = np.random.default_rng(n)
    x = 1.0 + rng.random((n, c)) * 0.01
    check("f32", x, out, 0.0)
    check("f32", x * np.where(np.arange(c) % 8 == 0, 1.0, 2.0 ** -13), out, 1e-6)
