"""What a decoder's layer refuses before it hands an address to a kernel."""
import pytest
import torch

from paper_2301_01333_amd import binding
from paper_2301_01333_amd.decoder import DecoderAttention, check_rows, check_weights

CPU = torch.device("cpu")


def test_rows_as_they_should_be():
    check_rows(torch.empty((5, 8, 64), dtype=torch.bfloat16), torch.bfloat16, 8, 64, CPU)
    check_rows(torch.empty((0, 8, 64)), torch.float32, 8, 64, CPU)
    check_rows(torch.empty((5, 11, 64))[:, 2:10], torch.float32, 8, 64, CPU)   # a slice: strides are the kernels' business
    check_rows(torch.empty((8, 5, 64)).transpose(0, 1), torch.float32, 8, 64, CPU)


@pytest.mark.parametrize("rows,dtype,device", [
    (torch.empty((5, 8, 64), dtype=torch.bfloat16), torch.float32, CPU),       # half the bytes that would be read
    (torch.empty((5, 8, 64), dtype=torch.float32), torch.bfloat16, CPU),
    (torch.empty((5, 7, 64)), torch.float32, CPU),
    (torch.empty((5, 9, 64)), torch.float32, CPU),
    (torch.empty((5, 8, 32)), torch.float32, CPU),
    (torch.empty((5, 8 * 64)), torch.float32, CPU),
    (torch.empty((1, 5, 8, 64)), torch.float32, CPU),
    (torch.empty(()), torch.float32, CPU),
    (torch.empty((5, 64, 8)).transpose(1, 2), torch.float32, CPU),
    (torch.empty((5, 8, 128))[:, :, ::2], torch.float32, CPU),
    (torch.empty((5, 8, 64)), torch.float32, torch.device("cuda", 0)),
])
def test_rows_that_are_not(rows, dtype, device):
    with pytest.raises(ValueError):
        check_rows(rows, dtype, 8, 64, device)


@pytest.mark.parametrize("weights", [
    (torch.ones(64), None), (None, torch.ones(64)), (torch.ones(64), torch.ones(32)), (torch.ones(64).bfloat16(), torch.ones(64).bfloat16()),
    (torch.ones(128)[::2], torch.ones(64)), (torch.ones((1, 64)), torch.ones((1, 64))),
])
def test_weights_that_are_none(weights):
    with pytest.raises(ValueError):
        check_weights(*weights, torch.float32, 64)
    with pytest.raises(ValueError):
        DecoderAttention("f32", 4, 2, 64, 1, 64, q_weight=weights[0], k_weight=weights[1])


def test_weights_of_both_or_of_neither():
    check_weights(None, None, torch.float32, 64)
    check_weights(torch.ones(64), torch.ones(64), torch.float32, 64)


def test_a_layer_of_another_type_or_with_weights_elsewhere():
    with pytest.raises(ValueError):
        DecoderAttention("i8", 4, 2, 64, 1, 64)
    with pytest.raises(ValueError):
        DecoderAttention("f32", 4, 2, 64, 1, 64, q_weight=torch.ones(64), k_weight=torch.ones(64))


@pytest.mark.gpu
def test_refused_calls_leave_the_layer_as_it_is():
    hq, hk, d = 4, 2, 64
    make = lambda n, **kw: torch.randn((n, hq + 2 * hk, d), device="cuda", **kw)  # noqa: E731
    block = DecoderAttention("f32", hq, hk, d, 2, 64)
    block.prefill(make(12), [7, 5])
    cache, lens = block.cache.clone(), block.lens.clone()
    for bad in (make(12, dtype=torch.bfloat16), make(12).cpu(), make(12)[:, 1:], make(12)[..., :32], make(12).transpose(1, 2)):
        with pytest.raises(ValueError):
            block.prefill(bad, [7, 5])
        with pytest.raises(ValueError):
            block.step(bad[:2])
    for lengths in ([13, -1], [12], [], [7, 6], [65, 1]):
        with pytest.raises(ValueError):
            block.prefill(make(max(sum(lengths), 0)), lengths) if lengths != [7, 6] else block.prefill(make(12), lengths)
    odd = torch.randn(12 * 8 * 64 + 1, device="cuda")[1:].view(12, 8, 64)
    for call in (lambda: block.prefill(odd, [7, 5]), lambda: block.step(odd[:2])):  # the library's own refusal
        with pytest.raises(binding.OgcError):
            call()
    torch.cuda.synchronize()
    assert torch.equal(block.cache, cache) and torch.equal(block.lens, lens) and block.held == 7
