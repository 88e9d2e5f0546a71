"""A decoder's projections in microscaled formats (include/ogc_mx.h) through the C ABI against oracle/mx.py in 64 bits.

Tolerances, derived from the arithmetic; H = finfo.eps / 2 is half a step of a type (bf16 2^-8, fp32 2^-24) relative to the value, 2^-134 and 2^-150 below
the normal numbers.
  written rows: exact (powers of two scale without rounding).  Gated and normed rows are rounded to the format from fp32 values that are off by R (below), so a
    value read back is half a step of the format off, 2^-4 |y| and 2^-10 of the scale (MX8), 1/4 |y| and 1/4 of the scale (MX4), and R; the scale is the one of some value
    within R of the largest.
  norm: the sum of c squares in at most 8 * ceil(c / 512) + 24 additions after one another, each 2^-24, of which the root halves the effect; root,
    reciprocal and two products 8 * 2^-24 more: R = (4 * ceil(c / 512) + 20) * 2^-24 * |y|.
  gate: the exponential's argument and its result 2^-22 together, the sum, the quotient and two products 2^-22 more: R = 2^-21 |y|.
  product: with A = sum |x| |w|, an fp32 sum is off by (k / 64 + 8) * 2^-24 * A.  The products of one instruction, 64 channels, are added with about 13 bits below the
    largest one kept (see ogc_mlp.h); products of two E2M1 values whose groups have equal scales need 8.  So MX8, or scales that differ: 64 * 2^-13 of the largest product of
    each instruction more."""
import numpy as np
import pytest

from oracle import mx
from paper_2301_01333_amd import binding

pytestmark = pytest.mark.gpu
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
TINY = {"bf16": 2.0 ** -134, "f32": 2.0 ** -150}
NAMES = {"mx4": binding.OGC_MX4, "mx8": binding.OGC_MX8}


def torch_():
    import torch

    return torch


def dt(name):
    torch = torch_()
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def stream():
    return int(torch_().cuda.current_stream().cuda_stream)


def device_rows(x, dtype, wide=None):
    """Device rows of the type, `wide` elements apart (the gap holds NaN), and their values in 64 bits."""
    torch = torch_()
    unit = 8 if dtype == "bf16" else 4
    wide = wide or mx.up(x.shape[1], unit)
    raw = torch.full((max(x.shape[0], 1), wide), float("nan"), dtype=dt(dtype), device="cuda")
    v = raw[:x.shape[0], :x.shape[1]]
    v.copy_(torch.from_numpy(np.asarray(x)).to(dt(dtype)))
    return v, v.double().cpu().numpy()


def sentinel(nbytes):
    return torch_().full((max(nbytes, 1) + 64,), 0xCD, dtype=torch_().uint8, device="cuda")


def empty_rows(n, c, dtype, wide=None):
    torch = torch_()
    unit = 8 if dtype == "bf16" else 4
    wide = wide or mx.up(c, unit) + unit
    raw = torch.empty((n + 1, wide), dtype=dt(dtype), device="cuda")
    raw.view(torch.uint8).fill_(0xCD)
    return raw, raw[:n, :c]


def only_inside(raw, n, c):
    """Nothing behind the rows' channels, and no row behind the last, was written."""
    torch = torch_()
    return bool((raw[:n, c:].contiguous().view(torch.uint8) == 0xCD).all() and (raw[n:].view(torch.uint8) == 0xCD).all())


def inside(got, want, tol, what):
    got = got.double().cpu().numpy() if hasattr(got, "cpu") else got
    with np.errstate(invalid="ignore"):
        bad = ~((np.abs(got - want) <= tol) | (np.isnan(want) & np.isnan(got)) | (got == want))
    if bad.any():
        i = np.unravel_index(int(np.where(bad, np.nan_to_num(np.abs(got - want) / (tol + 1e-300), nan=1e30), 0).argmax()), bad.shape)
        raise AssertionError("%s: %d of %d outside; worst at %s: got %g want %g tolerance %g" % (what, bad.sum(), bad.size, i, got[i], want[i], tol[i]))


def matrix_buffers(fmt, n, c):
    codes, scales = binding.ogc_mx_bytes(NAMES[fmt], n, c)
    return sentinel(codes), sentinel(scales), codes, scales


# ---- written and read back --------------------------------------------------------------------------------------------------
def write(fmt, dtype, x, wide=None):
    """(codes, scales) as numpy bytes after ogc_mx_write, checked for what must not have been written."""
    v, x64 = device_rows(x, dtype, wide)
    n, c = x.shape
    codes, scales, nc, ns = matrix_buffers(fmt, n, c)
    binding.ogc_mx_write(binding.mx_rows(binding.DTYPES[dtype], NAMES[fmt], n, c, 0, v.stride(0)), v.data_ptr(), codes.data_ptr(), scales.data_ptr(), stream())
    got, gots = codes.cpu().numpy(), scales.cpu().numpy()
    assert (got[nc:] == 0xCD).all() and (gots[ns:] == 0xCD).all()
    byte, _, scale = mx.places(n, c, NAMES[fmt])
    assert (got[byte[n:]] == 0xCD).all() and (gots[scale[n:]] == 0xCD).all()  # rounded-up rows stay as they were
    return got[:nc], gots[:ns], x64, codes, scales


def check_write(fmt, dtype, x, wide=None):
    print("case: write", fmt, dtype, x.shape, wide, flush=True)
    got, gots, x64, codes, scales = write(fmt, dtype, x, wide)
    n, c = x.shape
    pad = np.zeros((n, mx.up(c, 256)))
    pad[:, :c] = x64
    wantc, wante = mx.quantize(pad, NAMES[fmt])
    gotc, gote = mx.codes_of(got, gots, n, c, NAMES[fmt])
    assert np.array_equal(gote[:, ::32], wante)
    assert np.array_equal(gotc, wantc)
    for out in ("bf16", "f32"):
        raw, y = empty_rows(n, c, out)
        binding.ogc_mx_read(binding.mx_rows(binding.DTYPES[out], NAMES[fmt], n, c, 0, raw.stride(0)), codes.data_ptr(), scales.data_ptr(), y.data_ptr(), stream())
        want = mx.values(wantc, wante, NAMES[fmt])[:, :c]
        # exact but below the type's smallest number
        inside(y, want, np.where(np.abs(want) < 2.0 ** -126, TINY[out], 0.0), "read back as " + out)
        assert only_inside(raw, n, c)


@pytest.mark.parametrize("fmt", ["mx4", "mx8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,c", [(1, 1), (1, 32), (2, 31), (3, 33), (8, 256), (9, 257), (31, 100), (32, 640), (33, 1000), (70, 511), (5, 4100)])
def test_written_rows(fmt, dtype, n, c):
    rng = np.random.default_rng(n * 10000 + c)
    x = rng.normal(size=(n, c)) * np.exp(rng.normal(size=(n, 1)) * 4) * (1 + 30 * (rng.random((1, c)) < 0.05))
    check_write(fmt, dtype, x)
    check_write(fmt, dtype, x, mx.up(c, 8) + 24)


@pytest.mark.parametrize("fmt", ["mx4", "mx8"])
def test_written_rows_at_every_rounding(fmt):
    """Around every tie between codes, at scales over the whole range, from fp32; and the largest around every step of the scale."""
    table = mx.CODES[NAMES[fmt]]
    mid = (table[1:] + table[:-1]) / 2
    near = np.concatenate([table, mid, np.nextafter(mid.astype(np.float32), np.float32(0)), np.nextafter(mid.astype(np.float32), np.float32(1e9))])
    near = near[near < table[-1]]
    rows = []
    for e in list(range(-126, 118, 7)) + [-126, -125, -120, 117, 118]:
        for sign in (1, -1):
            for i in range(0, len(near), 31):
                g = np.zeros(32)
                g[:len(near[i:i + 31])] = near[i:i + 31]
                g[31] = table[-1]
                with np.errstate(over="ignore"):
                    rows.append(np.clip(sign * g * 2.0 ** e, -3.4e38, 3.4e38).astype(np.float32))
    edge = np.float32(7.0 if fmt == "mx4" else 464.0)
    for v in (edge, np.nextafter(edge, np.float32(0)), np.nextafter(edge, np.float32(1e9))):
        for e in range(-126, 117):
            g = np.linspace(0, 1, 32) * float(v)
            rows.append((g * 2.0 ** e).astype(np.float32))
    x = np.array(rows, dtype=np.float32)
    x = np.concatenate([x, np.zeros((-len(x) % 8, 32), np.float32)]).reshape(-1, 256)
    check_write(fmt, "f32", x)


@pytest.mark.parametrize("fmt", ["mx4", "mx8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_written_rows_at_the_ends(fmt, dtype):
    top = {"bf16": 3.3895313892515355e38, "f32": 3.4028234663852886e38}[dtype]
    x = np.zeros((9, 320))
    x[0, ::3] = top
    x[1, 5::40] = -top
    x[2] = 2.0 ** -149 if dtype == "f32" else 2.0 ** -133
    x[3, 0], x[3, 40], x[3, 70], x[3, 319] = np.inf, np.nan, -np.inf, np.inf
    x[4] = -0.0
    x[5, :] = np.linspace(-1, 1, 320) * 2.0 ** -126
    x[6, 100] = 1.76 * 2.0 ** 127
    x[7, 33], x[7, 34] = np.nan, 1.0
    x[8] = 1.0
    check_write(fmt, dtype, x)


def test_rows_beyond_4_gib():
    """Rows whose codes begin beyond 2^32 bytes."""
    torch = torch_()
    n, c = 1 << 18, 1 << 15
    codes, scales = binding.ogc_mx_bytes(1, n, c)
    assert codes > 1 << 32
    x = torch.zeros((n, c), dtype=torch.bfloat16, device="cuda")
    last = torch.from_numpy(np.random.default_rng(1).normal(size=(2, c))).to(torch.bfloat16).cuda()
    x[-2:] = last
    cb, sb = (torch.zeros(k, dtype=torch.uint8, device="cuda") for k in (codes, scales))
    d = binding.mx_rows(binding.OGC_BF16, 1, n, c, 0, c)
    binding.ogc_mx_write(d, x.data_ptr(), cb.data_ptr(), sb.data_ptr(), stream())
    x.fill_(7.0)
    binding.ogc_mx_read(d, cb.data_ptr(), sb.data_ptr(), x.data_ptr(), stream())
    want = mx.values(*mx.quantize(last.double().cpu().numpy(), 1), 1)
    inside(x[-2:], want, 0 * want, "last rows")
    assert not x[:-2].any()


def check_rounded(fmt, gotc, gote, y, R, c):
    """Values in a format, from fp32 values that are within R of y [n, c]."""
    n = y.shape[0]
    wide = mx.up(c, 256)
    pad, rad = np.zeros((n, wide)), np.zeros((n, wide))
    pad[:, :c], rad[:, :c] = y, R
    low, high = (mx.quantize(np.repeat(t.reshape(n, -1, 32).max(-1), 32, 1), NAMES[fmt])[1] for t in (np.maximum(np.abs(pad) - rad, 0), np.abs(pad) + rad))
    e = gote[:, ::32]
    assert ((e == low) | (e == high)).all()
    got = mx.values(gotc, e, NAMES[fmt])
    scale = np.repeat(np.where(e == 255, np.nan, np.exp2(e.astype(float) - 127)), 32, 1)
    tol = (np.abs(pad) / 16 + scale * 2.0 ** -10 if fmt == "mx8" else np.abs(pad) / 4 + scale / 4) + 1.1 * rad
    inside(got, np.where(np.isnan(scale), np.nan, pad), np.nan_to_num(tol), "rounded to " + fmt)
    assert not got[:, c:].any()


@pytest.mark.parametrize("fmt", ["mx4", "mx8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,c", [(1, 1), (3, 33), (33, 256), (20, 515), (7, 2000)])
def test_gated_rows(fmt, dtype, n, c):
    print("case: gate", fmt, dtype, n, c, flush=True)
    rng = np.random.default_rng(n + c)
    x = rng.normal(size=(n, 2 * c)) * 2
    x[0, 0], x[0, c // 2] = -80.0, 60.0
    v, x64 = device_rows(x, dtype, mx.up(2 * c, 8) + 8)
    codes, scales, nc, ns = matrix_buffers(fmt, n, c)
    binding.ogc_mx_write(binding.mx_rows(binding.DTYPES[dtype], NAMES[fmt], n, c, binding.OGC_GATE_SILU, v.stride(0)), v.data_ptr(), codes.data_ptr(), scales.data_ptr(), stream())
    y = mx.gated(x64[:, :c], x64[:, c:])
    gotc, gote = mx.codes_of(codes.cpu().numpy()[:nc], scales.cpu().numpy()[:ns], n, c, NAMES[fmt])
    check_rounded(fmt, gotc, gote, y, 2.0 ** -21 * np.abs(y), c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gate_of_the_largest_numbers(dtype):
    """|a| log2(e) is no fp32 number from |a| = 2.36e38 on; a * b / (1 + exp(-a)) is: a * b, or nothing."""
    x = np.zeros((2, 512))
    x[0, :256:4], x[1, :256:4] = 3.3e38, -3.3e38
    x[:, 1:256:4] = 2.0 ** 127
    x[:, 2:256:4] = -(2.0 ** 100)
    x[:, 3:256:4] = -88.0
    x[:, 256:] = np.random.default_rng(3).uniform(-0.5, 0.5, (2, 256)) * np.exp2(-np.repeat(np.arange(0, 128, 16), 32) / 4)
    v, x64 = device_rows(x, dtype)
    codes, scales, nc, ns = matrix_buffers("mx8", 2, 256)
    binding.ogc_mx_write(binding.mx_rows(binding.DTYPES[dtype], 1, 2, 256, 1, v.stride(0)), v.data_ptr(), codes.data_ptr(), scales.data_ptr(), stream())
    y = mx.gated(x64[:, :256], x64[:, 256:])
    gotc, gote = mx.codes_of(codes.cpu().numpy()[:nc], scales.cpu().numpy()[:ns], 2, 256, 1)
    assert (gote < 255).all()
    check_rounded("mx8", gotc, gote, y, 2.0 ** -21 * np.abs(y), 256)


def test_gate_of_what_is_no_number():
    x = np.zeros((1, 512))
    x[0, :256] = 1.0
    x[0, 256:] = 1.0
    x[0, 3], x[0, 40], x[0, 70], x[0, 256 + 100] = np.inf, -np.inf, np.nan, np.inf
    v, _ = device_rows(x, "f32")
    codes, scales, nc, ns = matrix_buffers("mx8", 1, 256)
    binding.ogc_mx_write(binding.mx_rows(0, 1, 1, 256, 1, v.stride(0)), v.data_ptr(), codes.data_ptr(), scales.data_ptr(), stream())
    _, e = mx.codes_of(codes.cpu().numpy()[:nc], scales.cpu().numpy()[:ns], 1, 256, 1)
    assert (e[0, ::32] == 255).tolist() == [True, True, True, True, False, False, False, False]


# ---- norm -------------------------------------------------------------------------------------------------------------------
def run_norm(dtype, n, c, out, residual, eps=1e-6, seed=0, alias=None, scale=1.0, x=None):
    torch = torch_()
    print("case: norm", dtype, n, c, out, residual, alias, flush=True)
    rng = np.random.default_rng(seed + n * 31 + c)
    unit = 8 if dtype == "bf16" else 4
    wide = mx.up(c, unit) + unit
    xv, x64 = device_rows(rng.normal(size=(n, c)) * scale if x is None else x, dtype, wide)
    rv, r64 = device_rows(rng.normal(size=(n, c)) * 3 * scale, dtype, wide + unit)
    w = torch.from_numpy(1 + 0.3 * rng.normal(size=c)).float().cuda()
    sraw, s = empty_rows(n, c, dtype)
    yraw, y = empty_rows(n, c, dtype)
    if alias == "sum is x":
        s = xv
    if alias == "sum is residual":
        s = rv
    if alias == "y is x":
        y = xv
    desc = binding.norm_desc(binding.DTYPES[dtype], n, c, {"same": 0, "mx4": 1, "mx8": 2}[out], eps, xv.stride(0), rv.stride(0), s.stride(0), y.stride(0))
    if out != "same":
        codes, scales, nc, ns = matrix_buffers(out, n, c)
    binding.ogc_norm_run(desc, xv.data_ptr(), rv.data_ptr() if residual else 0, w.data_ptr(), s.data_ptr() if residual else 0,
                         y.data_ptr() if out == "same" else codes.data_ptr(), 0 if out == "same" else scales.data_ptr(), stream())
    s64 = x64
    if residual:
        with np.errstate(over="ignore"):
            total = torch.from_numpy(x64.astype(np.float32) + r64.astype(np.float32)).to(dt(dtype))  # fp32 sum, rounded to the type
        s64 = total.double().numpy()
        assert np.array_equal(s.double().cpu().numpy(), s64, equal_nan=True)
    with np.errstate(invalid="ignore"):
        want = mx.norm(s64, w.double().cpu().numpy(), eps)
    R = (4 * -(-c // 512) + 20) * 2.0 ** -24 * np.abs(want)
    if out == "same":
        inside(y, want, HALF[dtype] * np.abs(want) + R + TINY[dtype], "norm")
        if alias is None:
            assert only_inside(yraw, n, c)
    else:
        assert (codes[nc:] == 0xCD).all() and (scales[ns:] == 0xCD).all()
        got, gots = codes.cpu().numpy()[:nc], scales.cpu().numpy()[:ns]
        byte, _, at = mx.places(n, c, NAMES[out])
        assert (got[byte[n:]] == 0xCD).all() and (gots[at[n:]] == 0xCD).all()
        check_rounded(out, *mx.codes_of(got, gots, n, c, NAMES[out]), want, R, c)
    if residual and alias is None:
        assert only_inside(sraw, n, c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("out", ["same", "mx4", "mx8"])
@pytest.mark.parametrize("n,c", [(1, 1), (1, 7), (3, 8), (9, 33), (2, 513), (33, 256), (5, 1531), (4, 4096), (17, 4097), (2, 8192), (1, 16384), (9, 9000), (1, 66000)])
def test_norm_shapes(dtype, out, n, c):
    for residual in (True, False):
        run_norm(dtype, n, c, out, residual)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("out,n,c", [("same", 2100, 100), ("same", 1500, 700), ("same", 1100, 4104), ("same", 1030, 9000), ("mx8", 8200, 300), ("mx8", 8211, 2048), ("mx4", 8193, 2304),
                                      ("mx8", 2049, 100), ("mx4", 2051, 513), ("mx8", 2055, 1030), ("mx8", 2100, 4096), ("mx4", 2049, 4100), ("mx8", 2052, 5000),
                                      ("mx8", 4100, 100), ("mx4", 4099, 513), ("mx8", 4111, 1030), ("mx8", 4097, 4096), ("mx4", 4097, 4100), ("mx8", 4098, 8192), ("mx8", 4099, 8200),
                                      ("mx4", 8193, 100), ("mx4", 8209, 513), ("mx8", 8195, 1030), ("same", 8195, 100), ("same", 8193, 256), ("same", 8200, 7), ("same", 8192, 257)])
def test_norm_of_many_rows(dtype, out, n, c):
    """Fewer wavefronts a row."""
    run_norm(dtype, n, c, out, True)


@pytest.mark.parametrize("alias", ["sum is x", "sum is residual", "y is x"])
@pytest.mark.parametrize("c", [100, 4096, 70000])
def test_norm_in_place(alias, c):
    for dtype in ("bf16", "f32"):
        run_norm(dtype, 3, c, "same", alias != "y is x", alias=alias)


def test_norm_ends():
    for eps in (0.0, 1e-6, 10.0):
        run_norm("f32", 3, 300, "same", True, eps=eps)
    run_norm("f32", 3, 300, "same", False, eps=0.0, scale=1e17)   # squares to 1e34 and their sum are fp32 numbers
    x = np.zeros((4, 64))
    x[1, 5], x[2, 6] = np.nan, np.inf
    x[3] = 1.0
    run_norm("bf16", 4, 64, "same", False, x=x)                   # zeros: zeros; NaN: NaN; an infinity: zeros and NaN, as the formula has it


# ---- product ----------------------------------------------------------------------------------------------------------------
def run_product(xf, dtype, m, n, k, bias=True, seed=0, x=None, w=None, spread=1.0, wide=None):
    """Matrices made by the oracle; rounded-up rows hold bytes that are no numbers."""
    torch = torch_()
    print("case: product", xf, dtype, m, n, k, bias, flush=True)
    rng = np.random.default_rng(seed + m + 7 * n + 13 * k)
    x = rng.normal(size=(m, k)) * np.exp(spread * rng.normal(size=(1, k))) if x is None else x
    w = rng.normal(size=(n, k)) / np.sqrt(k) if w is None else w
    dev, vals = [], []
    for v, fmt in ((x, xf), (w, "mx4")):
        c, s = mx.matrix(v, NAMES[fmt])
        byte, _, at = mx.places(v.shape[0], k, NAMES[fmt])
        c[byte[v.shape[0]:]], s[at[v.shape[0]:]] = 0xFF, 0xFF
        dev += [torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()]
        vals.append(mx.read(c, s, v.shape[0], k, NAMES[fmt]))
    b = torch.from_numpy(rng.normal(size=n)).float().cuda()
    raw, y = empty_rows(m, n, dtype, wide)
    desc = binding.mx_product_desc(binding.DTYPES[dtype], NAMES[xf], 0, m, n, k, int(bias), raw.stride(0))
    space = sentinel(max(binding.ogc_mx_product_workspace_bytes(desc), 16))
    binding.ogc_mx_product_run(desc, dev[0].data_ptr(), dev[1].data_ptr(), dev[2].data_ptr(), dev[3].data_ptr(), b.data_ptr() if bias else 0, y.data_ptr(),
                               space.data_ptr(), stream())
    x64, w64 = vals
    want = x64 @ w64.T + (b.double().cpu().numpy() if bias else 0.0)
    reach = np.abs(x64) @ np.abs(w64).T + (np.abs(b.double().cpu().numpy()) if bias else 0.0)
    tol = HALF[dtype] * np.abs(want) + (k / 64 + 8) * 2.0 ** -24 * reach + TINY[dtype]
    for first in range(0, k, 64):  # the largest product of 64 channels is at most the product of the largest
        tol = tol + 64 * 2.0 ** -13 * np.abs(x64[:, first:first + 64]).max(1)[:, None] * np.abs(w64[:, first:first + 64]).max(1)[None, :]
    inside(y, want, tol, "product")
    assert only_inside(raw, m, n)
    return y.double().cpu().numpy(), want, binding.ogc_mx_product_kernel_name(desc)


@pytest.mark.parametrize("xf", ["mx4", "mx8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 32, 32), (2, 33, 65), (31, 64, 256), (32, 100, 257), (33, 31, 1000), (65, 130, 300), (100, 257, 768), (130, 200, 520), (257, 300, 1024),
                                   (1, 1000, 4100), (40, 96, 2500)])
def test_product_shapes(xf, dtype, m, n, k):
    run_product(xf, dtype, m, n, k, bias=(m + n) % 2 == 0)


@pytest.mark.parametrize("xf", ["mx4", "mx8"])
@pytest.mark.parametrize("m,n,k", [(3, 70, 600), (70, 300, 1300), (300, 520, 512), (1290, 1300, 800), (3900, 3900, 704)])
def test_products_of_whole_numbers_are_exact(xf, m, n, k):
    """Scales of 1, whole numbers whose products and sums the instruction holds: every channel meets its own, once."""
    rng = np.random.default_rng(m)
    x = rng.choice([-6, -4, -3, -2, -1, 0, 1, 2, 3, 4, 6], size=(m, k)).astype(float)
    w = rng.choice([-6, -4, -3, -2, -1, 0, 1, 2, 3, 4, 6], size=(n, k)).astype(float)
    x[:, ::32], w[:, ::32] = (6.0 if xf == "mx4" else 448.0), 6.0  # (the largest of a group sets its scale to 1)
    if xf == "mx8":
        x[:, ::32] = 0.0  # scales of 2^-6 and so: still powers of two
    got, want, _ = run_product(xf, "f32", m, n, k, bias=False, x=x, w=w)
    assert np.array_equal(got, want)


@pytest.mark.parametrize("xf", ["mx4", "mx8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k,kernel", [
    (100, 90, 700, "few_kernel<%d, %d, 1, 1>"), (33, 8200, 300, "few_kernel<%d, %d, 1, 1>"), (33, 14300, 2100, "few_kernel<%d, %d, 2, 1>"), (300, 2000, 4000, "few_kernel<%d, %d, 2, 1>"),
    (255, 8000, 4100, "few_kernel<%d, %d, 2, 2>"), (317, 11383, 1700, "few_kernel<%d, %d, 2, 2>"),
    (401, 12765, 200, "tile_kernel<%d, %d, 2, 2, 2, 2>"), (354, 9393, 300, "tile_kernel<%d, %d, 2, 2, 2, 2>"), (226, 12461, 700, "tile_kernel<%d, %d, 2, 2, 2, 2>"),
    (162, 15797, 900, "tile_kernel<%d, %d, 2, 2, 2, 2>"), (788, 14543, 200, "tile_kernel<%d, %d, 2, 4, 4, 2>"), (1038, 11039, 300, "tile_kernel<%d, %d, 2, 4, 4, 2>"),
    (3900, 3900, 1700, "tile_kernel<%d, %d, 2, 4, 4, 2>"), (3841, 4001, 1300, "tile_kernel<%d, %d, 2, 4, 4, 2>")])
def test_product_by_kernel(xf, dtype, m, n, k, kernel):
    """Every kernel, with one stage of channels and with many, whole tiles and ragged ones."""
    _, _, name = run_product(xf, dtype, m, n, k, bias=k % 3 == 0)
    assert name == "ogc_mx_" + kernel % (binding.DTYPES[dtype], NAMES[xf])


@pytest.mark.parametrize("xf", ["mx4", "mx8"])
def test_product_scales(xf):
    """Groups whose scales are far apart; the largest and smallest scales; groups that are no numbers."""
    rng = np.random.default_rng(4)
    run_product(xf, "f32", 40, 40, 512, spread=6.0)
    x, w = rng.normal(size=(33, 300)), rng.normal(size=(35, 300))
    x[3] *= 2.0 ** 100
    x[4] *= 2.0 ** -100
    w[5] *= 2.0 ** 20
    w[6] *= 2.0 ** -20
    x[7, 40], w[8, 290] = np.nan, np.inf
    got, want, _ = run_product(xf, "f32", 33, 35, 300, x=x, w=w)
    assert np.isnan(got[7]).all() and np.isnan(got[:, 8]).all() and np.isnan(got).sum() == 35 + 33 - 1


def test_product_in_a_graph_and_on_a_stream_of_its_own():
    torch = torch_()
    rng = np.random.default_rng(9)
    m, n, k = 70, 96, 512
    mats = [mx.matrix(rng.normal(size=s), f) for s, f in (((m, k), 1), ((m, k), 1), ((n, k), 0))]
    x, xs = (torch.from_numpy(t).cuda() for t in mats[0])
    x2, xs2 = (torch.from_numpy(t).cuda() for t in mats[1])
    w, ws = (torch.from_numpy(t).cuda() for t in mats[2])
    desc = binding.mx_product_desc(1, 1, 0, m, n, k, 0, n)
    space = sentinel(binding.ogc_mx_product_workspace_bytes(desc))
    y, eager = (torch.zeros((m, n), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    run = lambda out: binding.ogc_mx_product_run(desc, x.data_ptr(), xs.data_ptr(), w.data_ptr(), ws.data_ptr(), 0, out.data_ptr(), space.data_ptr(), stream())  # noqa: E731
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        run(y)
    for i in range(4):
        if i == 2:
            x.copy_(x2)
            xs.copy_(xs2)
        y.fill_(3.0)
        g.replay()
        run(eager)
        torch.cuda.synchronize()
        assert torch.equal(y, eager) and not (y == 3.0).all()


@pytest.mark.parametrize("out", ["same", "mx8"])
def test_norm_beyond_4_gib(out):
    """Rows, and codes, that begin beyond 2^32 bytes."""
    torch = torch_()
    n, c = (1 << 18) + 3, 1 << 14
    x = torch.zeros((n, c), dtype=torch.bfloat16, device="cuda")
    last = torch.from_numpy(np.random.default_rng(2).normal(size=(3, c))).to(torch.bfloat16).cuda()
    x[-3:] = last
    weight, y = torch.ones(c, device="cuda"), torch.empty((n, c), dtype=torch.bfloat16, device="cuda")
    codes, scales = binding.ogc_mx_bytes(1, n, c)
    assert codes > 1 << 32
    cb, sb = (torch.zeros(k, dtype=torch.uint8, device="cuda") for k in (codes, scales))
    d = binding.norm_desc(binding.OGC_BF16, n, c, int(out == "mx8") * 2, 0.0, c, 0, 0, c)
    binding.ogc_norm_run(d, x.data_ptr(), 0, weight.data_ptr(), 0, y.data_ptr() if out == "same" else cb.data_ptr(), sb.data_ptr() if out != "same" else 0, stream())
    want = mx.norm(last.double().cpu().numpy(), 1.0, 0.0)
    if out != "same":
        binding.ogc_mx_read(binding.mx_rows(binding.OGC_BF16, 1, n, c, 0, c), cb.data_ptr(), sb.data_ptr(), y.data_ptr(), stream())
        top = np.repeat(np.abs(want).reshape(3, -1, 32).max(-1), 32, 1)
        inside(y[-3:], want, np.abs(want) * (2.0 ** -4 + 2.0 ** -20) + top * 2.0 ** -17, "last rows")
    else:
        inside(y[-3:], want, np.abs(want) * (2.0 ** -8 + 2.0 ** -20), "last rows")


@pytest.mark.parametrize("m,n,k", [(2, (1 << 18) + 70, 1 << 15), ((1 << 15) + 5, (1 << 15) + 256, 64)])
def test_products_beyond_4_gib(m, n, k):
    """Weights, or results, that begin beyond 2^32 bytes; the others are zeros."""
    torch = torch_()
    rng = np.random.default_rng(k)
    at = 33  # so many last rows of both
    xv, wv = (torch.zeros((r, k), dtype=torch.bfloat16, device="cuda") for r in (m, n))
    for v in (xv, wv):
        v[-at:] = torch.from_numpy(rng.normal(size=(min(at, v.shape[0]), k))).to(torch.bfloat16).cuda()
    mats = []
    for v, fmt in ((xv, 1), (wv, 0)):
        codes, scales = (torch.zeros(s, dtype=torch.uint8, device="cuda") for s in binding.ogc_mx_bytes(fmt, *v.shape))
        binding.ogc_mx_write(binding.mx_rows(binding.OGC_BF16, fmt, *v.shape, 0, k), v.data_ptr(), codes.data_ptr(), scales.data_ptr(), stream())
        mats.append((codes, scales, mx.values(*mx.quantize(v[-at:].double().cpu().numpy(), fmt), fmt)))
    (x, xs, x64), (w, ws, w64) = mats
    assert w.numel() > 1 << 32 or m * n * 4 > 1 << 32
    wide = mx.up(n, 4) + 4
    y = torch.full((m, wide), 5.0, device="cuda")
    binding.ogc_mx_product_run(binding.mx_product_desc(binding.OGC_F32, 1, 0, m, n, k, 0, wide), x.data_ptr(), xs.data_ptr(), w.data_ptr(), ws.data_ptr(), 0, y.data_ptr(), 0, stream())
    # (an instruction's 64 products: each 2^-13 of the largest at most; sums of k / 64 of them)
    tol = k * 2.0 ** -13 * np.abs(x64).max(1)[:, None] * np.abs(w64).max(1)[None, :] + (k / 64 + 8) * 2.0 ** -24 * (np.abs(x64) @ np.abs(w64).T)
    inside(y[-at:, n - at:n], x64 @ w64.T, tol, "last ones")
    assert not y[:-at, :n].any() and not y[-at:, :n - at].any() and bool((y[:, n:] == 5.0).all())


def test_products_at_once_on_two_streams():
    torch = torch_()
    rng = np.random.default_rng(12)
    m, n, k = 1400, 1300, 1000
    mats = [mx.matrix(rng.normal(size=s), 0) for s in ((m, k), (n, k))]
    (x, xs), (w, ws) = ([torch.from_numpy(t).cuda() for t in v] for v in mats)
    desc = binding.mx_product_desc(1, 0, 0, m, n, k, 0, 1304)
    ys = [torch.zeros((m, 1304), dtype=torch.bfloat16, device="cuda") for _ in range(5)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i, y in enumerate(ys[1:]):
        binding.ogc_mx_product_run(desc, x.data_ptr(), xs.data_ptr(), w.data_ptr(), ws.data_ptr(), 0, y.data_ptr(), 0, int(streams[i % 2].cuda_stream))
    torch.cuda.synchronize()
    binding.ogc_mx_product_run(desc, x.data_ptr(), xs.data_ptr(), w.data_ptr(), ws.data_ptr(), 0, ys[0].data_ptr(), 0, stream())
    assert ys[0].any() and all(torch.equal(y, ys[0]) for y in ys[1:])
