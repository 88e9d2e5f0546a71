"""The decoder's attention block at the ends of what its inputs may be.  Oracle and
tolerances: test_gpu_decoder.py."""
import numpy as np
import pytest

from test_gpu_decoder import torch_
from test_gpu_decoder_kernels import prompts, streams

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("qs,ks,causal", [([1], [33], 1), ([3], [33], 0), ([1, 70, 31], [1, 95, 63], 0), ([2, 40], [66, 129], 1)])
def test_prompt_infinite_last_values(dtype, d, many, qs, ks, causal):
    """A block of keys ends inside a unit, and the last value that there is holds infinities: they are the results of the rows that see it, and what
    follows the last key adds nothing to them."""
    torch = torch_()
    last = np.cumsum(ks) - 1

    def spoil(q, k, v):
        v[last, :, 3], v[last, :, d - 1] = float("inf"), float("-inf")

    kernel = "ogc_prompt_split_kernel<%d>" % (d // 32) if dtype == "f32" else streams(d) if many else "ogc_prompt_few_kernel<%d>" % (d // 32)
    o = prompts(kernel, dtype, qs, ks, 4, 2, d, d + sum(ks), causal=causal, spoil=spoil, copies=16 if many and dtype == "f32" else None)
    at = 0
    for a in qs:
        seen = o[at:at + a] if not causal else o[at + a - 1:at + a]
        assert (seen[..., 3] == float("inf")).all() and (seen[..., d - 1] == float("-inf")).all()
        assert torch.isfinite(o[at:at + a, :, 4:d - 1]).all() and (not causal or torch.isfinite(o[at:at + a - 1]).all())
        at += a
