"""A launch has at most 2^32 - 1 threads along an axis: what would need more is refused by the validation, what just fits is not."""
import os

import pytest

from paper_2301_01333_amd import binding as b

pytestmark = pytest.mark.skipif(not os.path.exists(b.LIB_PATH), reason="libogc_mlp.so not built (python -m paper_2301_01333_amd.build)")
SHAPE = -3
MOST = (1 << 24) - 1  # workgroups of 256 threads
P = 1 << 40           # an aligned address that nothing reads: the refusals come before any launch


def refused(call):
    with pytest.raises(b.OgcError) as e:
        call()
    assert e.value.status == SHAPE


def test_rope():
    def desc(tokens):
        return b.rope_desc(b.OGC_BF16, tokens, 1, 1, 32, 32, 0, 0, 0.0, 1.0, (32, 32), (32, 32), (32, 32), (32, 32))

    assert b.ogc_rope_validate(desc(4 * MOST)) == 0   # four tokens a workgroup
    for tokens in (4 * MOST + 1, (1 << 31) - 1):
        assert b.ogc_rope_validate(desc(tokens)) == SHAPE
        refused(lambda: b.ogc_rope_run(desc(tokens), *(8 * [P])))


def test_cache_rows():
    def args(heads, rows, most):
        return b.kv4_desc(heads, 32, 64, 9, 1, 4), b.kv4_rows(b.OGC_BF16, rows, most, (32, 32), (32, 32))

    # four wavefronts a workgroup, one for eight tokens of a head, and one more for an odd start
    for heads, rows in ((64, 8 * (MOST // 16 - 1)), (4, 8 * (MOST - 1)), (65536, 8 * 1022)):
        assert b.ogc_kv4_validate(*args(heads, rows, rows)) == 0
        assert b.ogc_kv4_validate(*args(heads, (1 << 31) - 1, rows)) == 0
        assert b.ogc_kv4_validate(*args(heads, rows + 16, rows + 16)) == SHAPE
        for call in (b.ogc_kv4_write, b.ogc_kv4_read):
            refused(lambda: call(*args(heads, (1 << 31) - 1, rows + 16), *(6 * [P])))


def test_cache_attention():
    def args(heads, group, rows, dtype=b.OGC_F32, keys=100):
        c = b.kv4_desc(heads, 32, 64, 9, 1, 4)
        return c, b.kv4_attention_desc(dtype, heads * group, rows, rows, keys, 0.125, (32, 32), (32, 32))

    assert b.ogc_kv4_attention_validate(*args(1, 1, 16 * MOST)) == 0
    assert b.ogc_kv4_attention_validate(*args(1, 1, 32 * MOST, b.OGC_BF16)) == 0
    assert b.ogc_kv4_attention_validate(*args(256, 16, MOST // 256)) == 0
    for a in (args(1, 1, 16 * MOST + 1), args(1, 1, 32 * MOST + 1, b.OGC_BF16), args(256, 16, MOST // 256 + 1)):
        assert b.ogc_kv4_attention_validate(*a) == SHAPE
        refused(lambda: b.ogc_kv4_attention_run(*a, *(8 * [P])))
        refused(lambda: b.ogc_kv4_attention_workspace_bytes(*a))


def test_prompts():
    def desc(batch, heads, rows, most):
        return b.prompt_desc(b.OGC_BF16, batch, heads, heads, 32, rows, 100, most, 100, 0.125, 1, (32, 32), (32, 32), (32, 32), (32, 32))

    assert b.ogc_prompt_validate(desc(1, 256, 128 * (MOST // 256), 128 * (MOST // 256))) == 0
    assert b.ogc_prompt_validate(desc(MOST, 1, 1 << 30, 128)) == 0
    for a in (desc(1, 256, 128 * (MOST // 256) + 1, 128 * (MOST // 256) + 1), desc(MOST + 1, 1, 1 << 30, 128), desc(1 << 20, 64, 1 << 20, 5)):
        assert b.ogc_prompt_validate(a) == SHAPE
        refused(lambda: b.ogc_prompt_run(a, *(6 * [P])))
