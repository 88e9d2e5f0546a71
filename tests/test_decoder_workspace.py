"""The workspace of attention over the 4-bit cache: what is asked for once is enough while the cache fills, and DecoderAttention's never moves."""
import os

import pytest

from paper_2301_01333_amd import binding as b

built = pytest.mark.skipif(not os.path.exists(b.LIB_PATH), reason="libogc_mlp.so not built (python -m paper_2301_01333_amd.build)")


@built
@pytest.mark.parametrize("batch,heads,group", [(1, 1, 1), (1, 8, 4), (3, 5, 2), (32, 8, 4), (48, 16, 1)])
@pytest.mark.parametrize("dtype", [b.OGC_F32, b.OGC_BF16])
def test_a_workspace_is_enough_for_fewer_tokens(batch, heads, group, dtype):
    d = 64
    cache = b.kv4_desc(heads, d, 64, 1 << 20, batch, 1 << 14)
    hq = heads * group
    last = 0
    for keys in sorted(list(range(1, 2600, 31)) + list(range(2600, 1 << 20, 12345)) + [768 * 128, 768 * 128 + 1, 1 << 20]):
        desc = b.kv4_attention_desc(dtype, hq, batch, 1, keys, 0.125, (hq * d, d), (hq * d, d))
        need = b.ogc_kv4_attention_workspace_bytes(cache, desc)
        assert need >= last, keys
        last = need


@pytest.mark.gpu
def test_the_layers_workspace_stays_where_it_is():
    """From lengths that one workgroup has to those that several share: a step that is on its way, or captured, keeps its workspace."""
    import numpy as np
    import torch

    from oracle import decoder
    from paper_2301_01333_amd.decoder import DecoderAttention
    from test_gpu_decoder import inside, tolerance

    hq, hk, d, n = 4, 2, 64, 1022
    g = torch.Generator(device="cuda").manual_seed(6)
    make = lambda n: torch.randn((n, hq + 2 * hk, d), generator=g, device="cuda")  # noqa: E731
    block = DecoderAttention("f32", hq, hk, d, 1, 1100)
    at = (block.workspace.data_ptr(), block.workspace.numel())
    block.prefill(make(n), [n])
    for s in range(6):
        qkv = make(1)
        q = block._turned(qkv, block.lens.clone())[0].double().cpu().numpy()
        o = block.step(qkv)
        assert (block.workspace.data_ptr(), block.workspace.numel()) == at
        data = decoder.Cache(block.cache.cpu().numpy().reshape(-1, hk, 2, 34 * d), hk, d, 64)
        count = n + s + 1
        k, v = (np.array([data.read(block.table[0].tolist(), t, which) for t in range(count)]) for which in (0, 1))
        want = decoder.attend(q, k, v, np.ones((1, count), dtype=bool), float(np.float32(d ** -0.5)))
        inside(o, want[0], tolerance("f32", *want, count, d), "step %d" % s)
