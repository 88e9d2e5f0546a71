"""Microscaled matrices and the operators around them on the host: the layout's arithmetic (csrc/ogc_mx_layout.h, compiled here) against the
documented order, oracle/mx.py against hand-worked cases, and the refusals of every entry point (found before any launch: no device is needed)."""
import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

from oracle import mx
from paper_2301_01333_amd import binding as b

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2301_01333_amd", "csrc")
built = pytest.mark.skipif(not os.path.exists(b.LIB_PATH), reason="libogc_mlp.so not built (python -m paper_2301_01333_amd.build)")
ARG, UNSUPPORTED, SHAPE, ALIGN, WORKSPACE = -1, -2, -3, -4, -5
P = 1 << 40  # an aligned address that nothing reads: every refusal comes before the launch

PROGRAM = r"""
#include "ogc_mx_layout.h"
#include <stdio.h>
#include <vector>
int main() {
    for (int format = 0; format < 2; ++format)
        for (int channels : {1, 256, 257, 800}) {
            const int rows = 70, c = mx_padded_channels(channels), r = (int)mx_padded_rows(rows);
            if (c % 256 || c < channels || c >= channels + 256 || r != 96) return printf("sizes\n"), 1;
            const int64_t bytes = mx_codes_of_32(format, c) * (r / 32);
            if (bytes != (int64_t)r * c / (format ? 1 : 2)) return printf("bytes\n"), 1;
            std::vector<int> seen(bytes, 0), scale((int64_t)r * c / 32, 0);
            const int per = format ? 16 : 32;
            for (int i = 0; i < r; ++i) {
                for (int j = 0; j < c; j += format ? 1 : 2) {
                    const int64_t at = ((int64_t)(i / 32) * (c / per) + j / per) * 512 + i % 32 * 16 + (format ? j % 16 : j % 32 / 2);
                    if (mx_code_at(format, c, i, j) != at) return printf("code %d %d\n", i, j), 1;
                    if (at < 0 || at >= bytes || seen[at]++) return printf("code %d %d out of range or twice\n", i, j), 1;
                }
                for (int g = 0; g < c / 32; ++g) {
                    const int64_t at = ((int64_t)(i / 32) * (c / 256) + g / 8) * 256 + g % 2 * 128 + i % 32 * 4 + g % 8 / 2;
                    if (mx_scales_at(c, i, g / 8, g % 2) + g % 8 / 2 != at) return printf("scale %d %d\n", i, g), 1;
                    if (at < 0 || at >= (int64_t)scale.size() || scale[at]++) return printf("scale %d %d out of range or twice\n", i, g), 1;
                }
            }
        }
    // beyond 2^32 bytes
    if (mx_code_at(1, 16384, 1 << 20, 16383) != (int64_t)(1 << 15) * 32 * 16384 + 1023 * 512 + 15) return printf("far code\n"), 1;
    if (mx_scales_at(1 << 20, (1 << 20) + 33, 4095, 1) != ((int64_t)(1 << 15) + 1) * (1 << 20) + 4095 * 256 + 128 + 4) return printf("far scale\n"), 1;
    puts("ok");
    return 0;
}
"""


def test_layout_is_the_documented_one_and_stays_in_range(tmp_path):
    src, exe = tmp_path / "layout.cpp", tmp_path / "layout"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-Wno-unused-function", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert (out.returncode, out.stdout.strip()) == (0, "ok")


# ---- the oracle ---------------------------------------------------------------------------------------------------------
def test_oracle_mx4_hand_cases():
    x = np.zeros((1, 64))
    x[0, :12] = [6.9, -0.25, 0.26, 0.75, 1.25, 1.26, -1.75, 2.5, 3.5, 5.0, 5.1, -0.1]   # scale 1: the largest rounds to 6
    x[0, 32:36] = [7.0, -1.0, 0.5, 0.51]                                                # 7 would round to 8: scale 2
    codes, e = mx.quantize(x, mx.MX4)
    assert e.tolist() == [[127, 128]]
    assert codes[0, :13].tolist() == [7, 8, 1, 2, 2, 3, 12, 4, 6, 6, 7, 8, 0]
    assert codes[0, 32:37].tolist() == [6, 9, 0, 1, 0]
    assert mx.values(codes, e, mx.MX4)[0, :6].tolist() == [6, -0.0, 0.5, 1, 1, 1.5]


def test_oracle_mx8_hand_cases():
    assert mx.E4M3[126] == 448 and mx.E4M3[1] == 2.0 ** -9 and mx.E4M3[8] == 2.0 ** -6 and (np.diff(mx.E4M3) > 0).all()
    x = np.zeros((1, 96))
    x[0, :8] = [464.0, -432.0, 1.0, 1.0625, 1.1875, -2.0 ** -10, 1.5 * 2.0 ** -9, 2.6 * 2.0 ** -9]  # scale 1: 464 is a tie that goes to 448
    x[0, 32:34] = [464.0001, 448.0]                                                                  # scale 2
    x[0, 64] = 2.0 ** -140                                                                           # scale 2^-127 at least
    codes, e = mx.quantize(x, mx.MX8)
    assert e.tolist() == [[127, 128, 0]]
    # 432 between 416 (1.625) and 448 (1.75): even mantissa 6; 1.0625 between 1 and 1.125: 1; 1.1875 between 1.125 and 1.25: 1.25
    assert mx.values(codes, e, mx.MX8)[0, :8].tolist() == [448, -448, 1, 1, 1.25, -0.0, 2 * 2.0 ** -9, 3 * 2.0 ** -9]
    assert mx.values(codes, e, mx.MX8)[0, 32:34].tolist() == [480, 448] and codes[0, 64] == 0  # 232.00005 is above the middle of 224 and 240


@pytest.mark.parametrize("fmt", [mx.MX4, mx.MX8])
def test_oracle_borders_and_bytes(fmt):
    for v, last in ((2.0 ** 127 * 1.99, mx.LAST[fmt]), (0.0, 0)):
        codes, e = mx.quantize(np.full((1, 32), v), fmt)
        assert e[0, 0] == last and np.isfinite(mx.values(codes, e, fmt)).all()
    for v in (np.inf, -np.inf, np.nan):
        x = np.ones((1, 64))
        x[0, 40] = v
        codes, e = mx.quantize(x, fmt)
        assert e[0, 1] == 255 and e[0, 0] != 255 and not codes[0, 32:].any() and np.isnan(mx.values(codes, e, fmt)[0, 32:]).all()
    rng = np.random.default_rng(3)
    x = rng.normal(size=(37, 300)) * np.exp(rng.normal(size=(37, 1)) * 3)
    data, scales = mx.matrix(x, fmt)
    assert (len(data), len(scales)) == (64 * 512 // (2 if fmt == mx.MX4 else 1), 64 * 16)
    got = mx.read(data, scales, 37, 300, fmt)
    pad = np.zeros((37, 320))
    pad[:, :300] = x
    want = mx.values(*mx.quantize(pad, fmt), fmt)[:, :300]
    assert np.array_equal(got, want)
    top = np.repeat(np.abs(pad).reshape(37, 10, 32).max(-1), 32, axis=1)[:, :300]
    assert (np.abs(got - x) <= (np.abs(x) / 4 + top / 8 if fmt == mx.MX4 else np.abs(x) / 16 + top * 2.0 ** -17)).all()


def test_oracle_sample_hand_cases():
    x = np.log([0.1, 0.4, 0.3, 0.2])
    for u, token in ((0.0, 0), (0.0999, 0), (0.1001, 1), (0.4999, 1), (0.5001, 2), (0.8001, 3), (0.99999, 3), (1.0, 3), (-3.0, 0), (np.nan, 0)):
        assert mx.sample(x, uniform=u)[0] == token, u
    assert abs(mx.sample(x, uniform=0.3)[1] - math_log(0.4)) < 1e-12
    for kw, kept in ((dict(top_k=1), {1}), (dict(top_k=2), {1, 2}), (dict(top_p=0.39), {1}), (dict(top_p=0.41), {1, 2}), (dict(top_p=0.71), {1, 2, 3}), (dict(top_p=0.0), {1}),
                     (dict(min_p=0.51), {1, 2}), (dict(min_p=0.49), {1, 2, 3}), (dict(min_p=2.0), {1}), (dict(top_k=3, top_p=0.44), {1}), (dict(top_k=3, top_p=0.45), {1, 2}),
                     (dict(temperature=0.0), {1}), (dict(temperature=float("nan")), {1}), (dict(temperature=0.01), {1})):
        assert {mx.sample(x, uniform=u, **kw)[0] for u in np.linspace(0, 0.999, 41)} == kept, kw
    ties = np.array([1.0, 3.0, 3.0, 2.0, 3.0, -0.0, 0.0])
    assert {mx.sample(ties, top_k=2, uniform=u)[0] for u in (0.1, 0.9)} == {1, 2}
    assert {mx.sample(ties, top_k=6, uniform=u)[0] for u in np.linspace(0, 0.9999, 3000)} == {0, 1, 2, 3, 4, 5}  # -0 and 0 are equal: the lower index
    assert mx.sample(np.full(5, -np.inf))[:2] == (-1, -np.inf) and mx.sample(np.full(5, np.nan))[0] == -1
    assert mx.sample(np.array([0.0, np.inf, 1.0, np.inf]), uniform=0.6)[0] == 3


def math_log(x):
    return float(np.log(x))


# ---- refusals -------------------------------------------------------------------------------------------------------------
def norm(**kw):
    a = dict(dtype=b.OGC_BF16, rows=5, channels=100, out=b.OGC_NORM_SAME, eps=1e-6, x_stride=104, residual_stride=104, sum_stride=104, y_stride=104)
    a.update(kw)
    return b.norm_desc(**a)


def rows(**kw):
    a = dict(dtype=b.OGC_BF16, fmt=b.OGC_MX8, rows=5, channels=100, gate=0, stride=208)
    a.update(kw)
    return b.mx_rows(**a)


def product(**kw):
    a = dict(dtype=b.OGC_BF16, x_format=b.OGC_MX8, w_format=b.OGC_MX4, m=5, n=100, k=300, has_bias=1, y_stride=104)
    a.update(kw)
    return b.mx_product_desc(**a)


def sample(**kw):
    a = dict(dtype=b.OGC_BF16, rows=3, vocab=1000, stride=1001)
    a.update(kw)
    return b.sample_desc(**a)


def refuses(status, call, *args):
    with pytest.raises(b.OgcError) as e:
        call(*args)
    assert e.value.status == status


TYPES = [(dict(dtype=b.OGC_F32), 0), (dict(dtype=b.OGC_I8), UNSUPPORTED), (dict(dtype=b.OGC_F8), UNSUPPORTED), (dict(dtype=4), ARG), (dict(dtype=-1), ARG)]


def strides(name):
    return [({name: s}, st) for s, st in ((-8, ALIGN), (108, ALIGN), (0, 0), (1 << 40, 0))]


@built
@pytest.mark.parametrize("kw,status", TYPES + [
    ({}, 0), (dict(out=1), 0), (dict(out=2), 0), (dict(out=3), ARG), (dict(out=-1), ARG), (dict(eps=-1.0), ARG), (dict(eps=float("nan")), ARG), (dict(eps=float("inf")), ARG),
    (dict(eps=0.0), 0), (dict(rows=0), 0), (dict(rows=-1), SHAPE), (dict(rows=1 << 22), SHAPE), (dict(channels=0), SHAPE), (dict(channels=1), 0), (dict(channels=(1 << 20) + 1), SHAPE),
    (dict(channels=1 << 20), 0), (dict(out=1, y_stride=3), 0),
] + strides("x_stride") + strides("residual_stride") + strides("sum_stride") + strides("y_stride"))
def test_norm_refusals(kw, status):
    assert b.ogc_norm_validate(norm(**kw)) == status
    if status:
        refuses(status, b.ogc_norm_run, norm(**kw), P, P, P, P, P, P)


@built
def test_norm_pointers():
    for out, needed in ((0, (0, 2, 3, 4)), (2, (0, 2, 3, 4, 5))):
        for at in needed:  # x, residual, weight, sum, y, scales
            args = 6 * [P]
            args[at] = 0
            refuses(ARG, b.ogc_norm_run, norm(out=out), *args)
        for at in range(6 if out else 5):
            args = 6 * [P]
            args[at] = P + 8
            refuses(ALIGN, b.ogc_norm_run, norm(out=out), *args)
    b.ogc_norm_run(norm(rows=0), 0, 0, 0, 0, 0)


@built
@pytest.mark.parametrize("kw,status", TYPES + [
    ({}, 0), (dict(fmt=0), 0), (dict(fmt=2), ARG), (dict(fmt=-1), ARG), (dict(gate=1), 0), (dict(gate=2), ARG), (dict(rows=0), 0), (dict(rows=-1), SHAPE), (dict(channels=0), SHAPE),
    (dict(channels=(1 << 20) + 1), SHAPE), (dict(rows=1 << 30), SHAPE), (dict(rows=1 << 24, channels=8192), SHAPE), (dict(rows=1 << 18, channels=1 << 16), 0),
] + strides("stride"))
def test_rows_refusals(kw, status):
    assert b.ogc_mx_validate(rows(**kw)) == status
    if status:
        refuses(status, b.ogc_mx_write, rows(**kw), P, P, P)
        refuses(status, b.ogc_mx_read, rows(**kw), P, P, P)


@built
def test_rows_pointers_and_sizes():
    for call in (b.ogc_mx_write, b.ogc_mx_read):
        for at in range(3):
            args = 3 * [P]
            args[at] = 0
            refuses(ARG, call, rows(), *args)
            args[at] = P + 8
            refuses(ALIGN, call, rows(), *args)
        call(rows(rows=0), 0, 0, 0)
    refuses(ARG, b.ogc_mx_read, rows(gate=1), P, P, P)
    assert b.ogc_mx_bytes(0, 33, 257) == (64 * 512 // 2, 64 * 16) and b.ogc_mx_bytes(1, 33, 257) == (64 * 512, 64 * 16) and b.ogc_mx_bytes(1, 0, 5) == (0, 0)
    assert b.ogc_mx_bytes(1, 1 << 30, 1 << 20) == (1 << 50, 1 << 45)
    for args, status in (((2, 1, 1), ARG), ((-1, 1, 1), ARG), ((0, -1, 1), SHAPE), ((0, 1, 0), SHAPE), ((0, 1, (1 << 20) + 1), SHAPE)):
        refuses(status, b.ogc_mx_bytes, *args)


@built
@pytest.mark.parametrize("kw,status", TYPES + [
    ({}, 0), (dict(x_format=0), 0), (dict(x_format=2), ARG), (dict(w_format=1), UNSUPPORTED), (dict(w_format=-1), ARG), (dict(has_bias=2), ARG), (dict(m=0), 0), (dict(m=-1), SHAPE),
    (dict(n=0), SHAPE), (dict(k=0), SHAPE), (dict(k=(1 << 20) + 1), SHAPE), (dict(k=1 << 20), 0), (dict(m=1 << 30), SHAPE), (dict(n=1 << 30), SHAPE), (dict(m=1 << 20, n=1 << 18), 0),
] + strides("y_stride"))
def test_product_refusals(kw, status):
    assert b.ogc_mx_product_validate(product(**kw)) == status
    assert bool(b.ogc_mx_product_kernel_name(product(**kw))) == (status == 0)
    if status:
        refuses(status, b.ogc_mx_product_run, product(**kw), *(7 * [P]))
        refuses(status, b.ogc_mx_product_workspace_bytes, product(**kw))


@built
def test_product_pointers():
    for at in range(6):  # x, scales, w, scales, bias, y
        args = 7 * [P]
        args[at] = 0
        refuses(ARG, b.ogc_mx_product_run, product(), *args)
        args[at] = P + 2
        refuses(ALIGN, b.ogc_mx_product_run, product(), *args)
    b.ogc_mx_product_run(product(m=0), *(7 * [0]))


@built
@pytest.mark.parametrize("kw,status", TYPES + [
    ({}, 0), (dict(rows=0), 0), (dict(rows=-1), SHAPE), (dict(rows=65536), SHAPE), (dict(vocab=0), SHAPE), (dict(vocab=1 << 20, stride=1 << 20), 0),
    (dict(vocab=(1 << 20) + 1, stride=1 << 21), SHAPE), (dict(stride=999), SHAPE), (dict(stride=1000), 0), (dict(stride=-1000), SHAPE),
])
def test_sample_refusals(kw, status):
    assert b.ogc_sample_validate(sample(**kw)) == status
    if status:
        refuses(status, b.ogc_sample_run, sample(**kw), *(9 * [P]))
        refuses(status, b.ogc_sample_workspace_bytes, sample(**kw))


@built
def test_sample_pointers():
    for at, name in enumerate(("logits", "temperature", "top_k", "top_p", "min_p", "uniform", "tokens", "log_probabilities")):
        args = 9 * [P]
        if name in ("logits", "uniform", "tokens"):
            args[at] = 0
            refuses(ARG, b.ogc_sample_run, sample(), *args)
        args[at] = P + (1 if name == "logits" else 2)
        refuses(ALIGN, b.ogc_sample_run, sample(), *args)
    refuses(ALIGN, b.ogc_sample_run, sample(dtype=b.OGC_F32), P + 2, *(8 * [P]))
    refuses(WORKSPACE, b.ogc_sample_run, sample(), *(8 * [P]), 0)
    refuses(ALIGN, b.ogc_sample_run, sample(), *(8 * [P]), P + 8)
    assert b.ogc_sample_workspace_bytes(sample(rows=0)) == 0
    for rows, vocab in ((1, 1), (1, 1 << 20), (64, 128000), (65535, 100)):
        need = b.ogc_sample_workspace_bytes(sample(rows=rows, vocab=vocab, stride=vocab))
        assert rows * (vocab + 7) // 8 * 4 <= need <= rows * (vocab * 5 + 9000)
    b.ogc_sample_run(sample(rows=0), *(9 * [0]))


@built
def test_null_descriptions():
    l, none = b.lib(), [None]
    assert l.ogc_norm_validate(None) == ARG and l.ogc_mx_validate(None) == ARG and l.ogc_mx_product_validate(None) == ARG and l.ogc_sample_validate(None) == ARG
    assert l.ogc_norm_run(None, *(7 * none)) == ARG and l.ogc_mx_write(None, *(4 * none)) == ARG and l.ogc_mx_read(None, *(4 * none)) == ARG
    assert l.ogc_mx_product_run(None, *(8 * none)) == ARG and l.ogc_sample_run(None, *(10 * none)) == ARG
    size = ctypes.c_size_t()
    assert l.ogc_mx_bytes(0, 1, 1, None, size) == ARG and l.ogc_mx_bytes(0, 1, 1, size, None) == ARG
    assert l.ogc_mx_product_workspace_bytes(product(), None) == ARG and l.ogc_sample_workspace_bytes(sample(), None) == ARG
    assert l.ogc_mx_product_kernel_name(None) is None


@built
def test_reported_kernel_names_are_in_the_library():
    nm = shutil.which("nm") or "/opt/rocm/llvm/bin/llvm-nm"
    out = subprocess.run([nm, "-C", "--defined-only", b.LIB_PATH], check=True, capture_output=True, text=True).stdout
    kernels, seen = set(re.findall(r"\bvoid (ogc_\w+<[^>]*>)\(", out)), set()
    for dtype in (b.OGC_F32, b.OGC_BF16):
        for fmt in (b.OGC_MX4, b.OGC_MX8):
            for m in (1, 20, 40, 100, 300, 1000, 5000):
                for n in (64, 1000, 8192):
                    seen.add(b.ogc_mx_product_kernel_name(product(dtype=dtype, x_format=fmt, m=m, n=n, k=4096, y_stride=8192)))
    assert seen <= kernels


@built
def test_products_of_many_tiles():
    """A launch has fewer than 2^32 threads: beyond 2^24 tiles of 128 x 128 the large ones, whatever k, and beyond 2^23 of those none."""
    for k in (1, 256, 8192):
        assert "2, 4, 4, 2>" in b.ogc_mx_product_kernel_name(product(m=1 << 20, n=1 << 18, k=k))
    for m, n, status in ((1 << 21, 1 << 18, SHAPE), (1 << 21, (1 << 18) - 256, 0), ((1 << 21) + 1, 64, SHAPE), (64, (1 << 26) + 1, SHAPE), (64, 1 << 26, 0), (1 << 21, 1 << 26, SHAPE)):
        assert b.ogc_mx_product_validate(product(m=m, n=n, y_stride=1 << 26)) == status, (m, n)
