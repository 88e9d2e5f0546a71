"""The decoder's attention block on the host: the cache's layout arithmetic (csrc/ogc_kv4_layout.h, compiled here) against the documented
order, places out of range, and the refusals of every entry point (found before any launch: no device is needed)."""
import itertools
import os
import re
import shutil
import subprocess

import pytest

from paper_2301_01333_amd import binding as b

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2301_01333_amd", "csrc")

PROGRAM = r"""
#include "ogc_kv4_layout.h"
#include <stdio.h>
#include <vector>
int main() {
    for (int d = 32; d <= 128; d += 32) {
        const int bytes = kv4_record_bytes(d);
        std::vector<int> seen(2 * bytes, 0);  // half bytes
        for (int t = 0; t < 32; ++t)
            for (int c = 0; c < d; ++c) {
                // keys [token][channel / 2], values [channel / 32][token / 8][channel % 16][channel / 16 % 2][token % 8 / 2]
                const int k = t * (d / 2) + c / 2, v = 16 * d + (((c / 32 * 4 + t / 8) * 16 + c % 16) * 2 + c / 16 % 2) * 4 + t % 8 / 2;
                if (kv4_key_at(d, t, c / 8 * 8) + c % 8 / 2 != k) return printf("key %d %d %d\n", d, t, c), 1;
                if (kv4_value_at(d, t / 8, c) + t % 8 / 2 != v) return printf("value %d %d %d\n", d, t, c), 1;
                ++seen[2 * k + c % 2];
                ++seen[2 * v + t % 2];
            }
        for (int g = 0; g < d / 32; ++g)
            for (int t = 0; t < 32; ++t)
                for (int at : {kv4_key_scale_at(d, g, t), kv4_value_scale_at(d, g, t)}) {
                    ++seen[2 * at];
                    ++seen[2 * at + 1];
                }
        if (kv4_key_scale_at(d, 0, 0) != 32 * d || kv4_value_scale_at(d, 0, 0) != 33 * d) return printf("scales\n"), 1;
        for (int n : seen)
            if (n != 1) return printf("a half byte of %d channels belongs to %d values\n", d, n), 1;
    }
    // places of tokens: in the page table's page or nowhere, never outside the cache
    const int heads = 3, page = 64, pages = 7, d = 96, width = 4;
    const int64_t size = (int64_t)pages * heads * (page / 32) * kv4_record_bytes(d);
    const int32_t table[2][width] = {{6, 0, -1, 3}, {7, 2147483647, -2147483647 - 1, 5}};
    for (int row = 0; row < 2; ++row)
        for (int h = 0; h < heads; ++h)
            for (int t = 0; t < 2 * width * page; ++t) {
                const int64_t at = kv4_record_at(table[row], width, page, pages, heads, d, t, h);
                const int e = t / page, p = e < width ? table[row][e] : -1;
                const bool there = p >= 0 && p < pages;
                if (there != (at >= 0)) return printf("token %d of row %d\n", t, row), 1;
                if (there && (at != (((int64_t)p * heads + h) * (page / 32) + t % page / 32) * 34 * d || at + 34 * d > size || at % 16)) return printf("at\n"), 1;
            }
    // beyond 2^32 bytes
    const int32_t far[1] = {4000000};
    if (kv4_record_at(far, 1, 256, 4000001, 8, 128, 255, 7) != ((int64_t)4000000 * 8 + 7) * 8 * 4352 + 7 * 4352) return printf("far\n"), 1;
    puts("ok");
    return 0;
}
"""


def test_cache_layout_is_the_documented_one_and_stays_in_range(tmp_path):
    src, exe = tmp_path / "layout.cpp", tmp_path / "layout"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-Wno-unused-function", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert (out.returncode, out.stdout.strip()) == (0, "ok")


built = pytest.mark.skipif(not os.path.exists(b.LIB_PATH), reason="libogc_mlp.so not built (python -m paper_2301_01333_amd.build)")
ARG, UNSUPPORTED, SHAPE, ALIGN, WORKSPACE = -1, -2, -3, -4, -5
P = 1 << 40  # an aligned address that nothing reads: every refusal comes before the launch


def rope(**kw):
    a = dict(dtype=b.OGC_BF16, tokens=8, q_heads=4, kv_heads=2, head_dim=64, rot_dim=64, layout=0, norm=1, eps=1e-6, magnitude=1.0,
             q_stride=(512, 64), k_stride=(512, 64), qo_stride=(256, 64), ko_stride=(128, 64))
    a.update(kw)
    return b.rope_desc(**a)


def cache(**kw):
    a = dict(kv_heads=2, head_dim=64, page_size=64, pages=9, batch=3, table_width=4)
    a.update(kw)
    return b.kv4_desc(**a)


def rows(**kw):
    a = dict(dtype=b.OGC_BF16, rows=10, max_rows=5, k_stride=(128, 64), v_stride=(128, 64))
    a.update(kw)
    return b.kv4_rows(**a)


def asks(**kw):
    a = dict(dtype=b.OGC_BF16, q_heads=4, rows=3, max_rows=1, max_keys=200, scale=0.125, q_stride=(256, 64), o_stride=(256, 64))
    a.update(kw)
    return b.kv4_attention_desc(**a)


def prompt(**kw):
    a = dict(dtype=b.OGC_BF16, batch=2, q_heads=4, kv_heads=2, head_dim=64, q_rows=20, k_rows=30, max_q=15, max_k=20, scale=0.125, causal=1,
             q_stride=(256, 64), k_stride=(128, 64), v_stride=(128, 64), o_stride=(256, 64))
    a.update(kw)
    return b.prompt_desc(**a)


STRIDES = [((-64, 64), ALIGN), ((512, -64), ALIGN), ((516, 64), ALIGN), ((512, 68), ALIGN), ((0, 64), 0), ((512, 0), 0)]


@built
@pytest.mark.parametrize("kw,status", [
    ({}, 0), (dict(dtype=b.OGC_F32), 0), (dict(dtype=b.OGC_I8), UNSUPPORTED), (dict(dtype=b.OGC_F8), UNSUPPORTED), (dict(dtype=4), ARG), (dict(dtype=-1), ARG),
    (dict(tokens=0), 0), (dict(tokens=-1), SHAPE), (dict(q_heads=0), SHAPE), (dict(kv_heads=0), SHAPE),
    (dict(head_dim=0), SHAPE), (dict(head_dim=48, rot_dim=48), UNSUPPORTED), (dict(head_dim=160), UNSUPPORTED), (dict(head_dim=128), 0),
    (dict(rot_dim=0), 0), (dict(rot_dim=8), 0), (dict(rot_dim=20), UNSUPPORTED), (dict(rot_dim=72), SHAPE), (dict(rot_dim=-8), SHAPE),
    (dict(layout=1), 0), (dict(layout=2), ARG), (dict(norm=2), ARG), (dict(eps=-1.0), ARG), (dict(eps=float("nan")), ARG), (dict(norm=0, eps=-1.0), 0),
    (dict(magnitude=float("inf")), ARG), (dict(magnitude=0.0), 0),
] + [({which: s}, st) for which in ("q_stride", "k_stride", "qo_stride", "ko_stride") for s, st in STRIDES])
def test_rope_refusals(kw, status):
    assert b.ogc_rope_validate(rope(**kw)) == status
    if status:
        with pytest.raises(b.OgcError) as e:
            b.ogc_rope_run(rope(**kw), P, P, P, P, P, P, P, P)
        assert e.value.status == status


@built
@pytest.mark.parametrize("at,ptr,status", [(i, 0, ARG) for i in range(8)] + [(i, P + 8, ALIGN) for i in (0, 1, 2, 3, 6, 7)] + [(4, P + 2, ALIGN), (5, P + 4, ALIGN)])
def test_rope_pointers(at, ptr, status):
    args = 8 * [P]
    args[at] = ptr
    with pytest.raises(b.OgcError) as e:
        b.ogc_rope_run(rope(), *args)
    assert e.value.status == status


CACHES = [(dict(kv_heads=0), SHAPE), (dict(head_dim=0), SHAPE), (dict(head_dim=80), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED), (dict(page_size=0), SHAPE),
          (dict(page_size=48), SHAPE), (dict(page_size=16), SHAPE), (dict(pages=0), SHAPE), (dict(batch=0), SHAPE), (dict(batch=65536), SHAPE),
          (dict(table_width=0), SHAPE), (dict(table_width=1 << 25), SHAPE), (dict(page_size=1 << 30, table_width=2), SHAPE), (dict(pages=1 << 30), 0)]


@built
@pytest.mark.parametrize("kw,status", CACHES)
def test_cache_refusals(kw, status):
    c = cache(**kw)
    assert b.ogc_kv4_validate(c, rows()) == status
    assert b.ogc_kv4_attention_validate(c, asks()) == status
    if status:
        for call in (lambda: b.ogc_kv4_cache_bytes(c), lambda: b.ogc_kv4_write(c, rows(), P, P, P, P, P, P), lambda: b.ogc_kv4_read(c, rows(), P, P, P, P, P, P),
                     lambda: b.ogc_kv4_attention_run(c, asks(), P, P, P, P, P, P, P), lambda: b.ogc_kv4_attention_workspace_bytes(c, asks())):
            with pytest.raises(b.OgcError) as e:
                call()
            assert e.value.status == status


@built
def test_cache_bytes():
    assert b.ogc_kv4_cache_bytes(cache()) == 9 * 2 * 2 * 34 * 64
    assert b.ogc_kv4_cache_bytes(cache(pages=1 << 24, head_dim=128, page_size=256, kv_heads=8)) == (1 << 24) * 8 * 8 * 34 * 128


@built
@pytest.mark.parametrize("kw,status", [
    ({}, 0), (dict(dtype=b.OGC_F32), 0), (dict(dtype=b.OGC_I8), UNSUPPORTED), (dict(dtype=9), ARG), (dict(rows=-1), SHAPE), (dict(max_rows=-1), SHAPE), (dict(rows=0), 0),
] + [({which: s}, st) for which in ("k_stride", "v_stride") for s, st in STRIDES])
def test_rows_refusals(kw, status):
    assert b.ogc_kv4_validate(cache(), rows(**kw)) == status
    if status:
        for call in (lambda: b.ogc_kv4_write(cache(), rows(**kw), P, P, P, P, P, P), lambda: b.ogc_kv4_read(cache(), rows(**kw), P, P, P, P, P, P)):
            with pytest.raises(b.OgcError) as e:
                call()
            assert e.value.status == status


@built
@pytest.mark.parametrize("at", range(6))
def test_write_and_read_pointers(at):
    args = 6 * [P]
    args[at] = 0
    for call in (b.ogc_kv4_write, b.ogc_kv4_read):
        with pytest.raises(b.OgcError) as e:
            call(cache(), rows(), *args)
        assert e.value.status == ARG
        odd = 6 * [P]
        odd[at] = P + 2
        with pytest.raises(b.OgcError) as e:
            call(cache(), rows(), *odd)
        assert e.value.status == ALIGN


@built
@pytest.mark.parametrize("kw,status", [
    ({}, 0), (dict(dtype=b.OGC_F32), 0), (dict(dtype=b.OGC_I8), UNSUPPORTED), (dict(dtype=-3), ARG), (dict(q_heads=0), SHAPE), (dict(q_heads=3), SHAPE), (dict(q_heads=514), SHAPE),
    (dict(q_heads=512), 0), (dict(rows=-1), SHAPE), (dict(max_rows=-1), SHAPE), (dict(max_keys=-1), SHAPE), (dict(max_keys=0), 0), (dict(rows=0), 0),
    (dict(scale=0.0), ARG), (dict(scale=-1.0), ARG), (dict(scale=float("nan")), ARG), (dict(scale=float("inf")), ARG), (dict(scale=2.0 ** 61), ARG), (dict(scale=2.0 ** 60), 0),
] + [({which: s}, st) for which in ("q_stride", "o_stride") for s, st in STRIDES])
def test_cache_attention_refusals(kw, status):
    assert b.ogc_kv4_attention_validate(cache(), asks(**kw)) == status
    if status:
        with pytest.raises(b.OgcError) as e:
            b.ogc_kv4_attention_run(cache(), asks(**kw), P, P, P, P, P, P, P)
        assert e.value.status == status


@built
@pytest.mark.parametrize("at", range(6))
def test_cache_attention_pointers(at):
    args = 6 * [P]
    args[at] = 0
    with pytest.raises(b.OgcError) as e:
        b.ogc_kv4_attention_run(cache(), asks(), *args, P)
    assert e.value.status == ARG
    args[at] = P + 2
    with pytest.raises(b.OgcError) as e:
        b.ogc_kv4_attention_run(cache(), asks(), *args, P)
    assert e.value.status == ALIGN


@built
def test_cache_attention_workspace():
    c = cache(table_width=512, batch=1)
    need = b.ogc_kv4_attention_workspace_bytes(c, asks(max_keys=30000))
    assert need > 0  # one short batch of long sequences is shared
    for ws, status in ((0, WORKSPACE), (P + 8, ALIGN)):
        with pytest.raises(b.OgcError) as e:
            b.ogc_kv4_attention_run(c, asks(max_keys=30000), P, P, P, P, P, P, ws)
        assert e.value.status == status
    assert b.ogc_kv4_attention_workspace_bytes(c, asks(max_keys=0)) == 0
    assert b.ogc_kv4_attention_workspace_bytes(c, asks(rows=0)) == 0


@built
@pytest.mark.parametrize("kw,status", [
    ({}, 0), (dict(dtype=b.OGC_F32), 0), (dict(dtype=b.OGC_I8), UNSUPPORTED), (dict(dtype=5), ARG), (dict(batch=0), SHAPE), (dict(q_heads=0), SHAPE), (dict(kv_heads=0), SHAPE),
    (dict(q_heads=5), SHAPE), (dict(q_heads=1024), SHAPE), (dict(head_dim=0), SHAPE), (dict(head_dim=72), UNSUPPORTED), (dict(head_dim=192), UNSUPPORTED),
    (dict(q_rows=-1), SHAPE), (dict(k_rows=-1), SHAPE), (dict(max_q=-1), SHAPE), (dict(max_k=-1), SHAPE), (dict(q_rows=0), 0), (dict(k_rows=0), 0),
    (dict(q_rows=1 << 30, max_q=1 << 30, k_rows=1 << 30), SHAPE), (dict(q_rows=1 << 29, max_q=1 << 29, k_rows=(1 << 31) - 1), SHAPE),
    (dict(scale=0.0), ARG), (dict(scale=float("-inf")), ARG), (dict(scale=2.0 ** -61), ARG), (dict(causal=0), 0), (dict(causal=2), ARG),
] + [({which: s}, st) for which in ("q_stride", "k_stride", "v_stride", "o_stride") for s, st in STRIDES])
def test_prompt_refusals(kw, status):
    assert b.ogc_prompt_validate(prompt(**kw)) == status
    assert bool(b.ogc_prompt_kernel_name(prompt(**kw))) == (status == 0)
    if status:
        with pytest.raises(b.OgcError) as e:
            b.ogc_prompt_run(prompt(**kw), P, P, P, P, P, P)
        assert e.value.status == status


@built
@pytest.mark.parametrize("at", range(6))
def test_prompt_pointers(at):
    args = 6 * [P]
    args[at] = 0
    with pytest.raises(b.OgcError) as e:
        b.ogc_prompt_run(prompt(), *args)
    assert e.value.status == ARG
    args[at] = P + 2
    with pytest.raises(b.OgcError) as e:
        b.ogc_prompt_run(prompt(), *args)
    assert e.value.status == ALIGN


@built
def test_calls_without_rows_do_nothing():
    """(no device here: a launch would fail)"""
    b.ogc_rope_run(rope(tokens=0), 0, 0, 0, 0, 0, 0, 0, 0)
    b.ogc_kv4_write(cache(), rows(rows=0), 0, 0, 0, 0, 0, 0)
    b.ogc_kv4_read(cache(), rows(max_rows=0), 0, 0, 0, 0, 0, 0)
    b.ogc_kv4_attention_run(cache(), asks(rows=0), 0, 0, 0, 0, 0, 0, 0)
    b.ogc_prompt_run(prompt(q_rows=0), 0, 0, 0, 0, 0, 0)


@built
def test_null_descriptions_are_refused():
    l = b.lib()
    none = [None]
    assert l.ogc_rope_validate(None) == ARG and l.ogc_prompt_validate(None) == ARG
    assert l.ogc_kv4_validate(None, rows()) == ARG and l.ogc_kv4_validate(cache(), None) == ARG
    assert l.ogc_kv4_attention_validate(None, asks()) == ARG and l.ogc_kv4_attention_validate(cache(), None) == ARG
    assert l.ogc_kv4_cache_bytes(cache(), None) == ARG and l.ogc_kv4_attention_workspace_bytes(cache(), asks(), None) == ARG
    assert l.ogc_rope_run(None, *(9 * none)) == ARG and l.ogc_prompt_run(None, *(7 * none)) == ARG
    assert l.ogc_kv4_write(None, None, *(7 * none)) == ARG and l.ogc_kv4_attention_run(None, None, *(8 * none)) == ARG


@built
def test_reported_kernel_names_are_in_the_library():
    nm = shutil.which("nm") or "/opt/rocm/llvm/bin/llvm-nm"
    out = subprocess.run([nm, "-C", "--defined-only", b.LIB_PATH], check=True, capture_output=True, text=True).stdout
    kernels, seen = set(re.findall(r"\bvoid (ogc_\w+<[^>]*>)\(", out)), set()
    for dtype, d, wide in itertools.product((b.OGC_F32, b.OGC_BF16), (32, 64, 96, 128), (False, True)):
        stride = ((1 << 26) if wide else 2 * d, d)  # (a token's stride too wide for 32 bits of offset)
        seen.add(b.ogc_prompt_kernel_name(prompt(dtype=dtype, head_dim=d, k_stride=stride, v_stride=stride)))
    many = 1 << 14
    for d in (32, 64, 96, 128):
        seen.add(b.ogc_prompt_kernel_name(prompt(head_dim=d, q_rows=many, max_q=many, k_rows=many, max_k=many)))
    assert len(seen) == 20 and seen <= kernels
