"""oracle/decoder.py against hand-worked cases and second definitions."""
import numpy as np
import torch

from oracle import decoder


def test_quantize_hand_cases():
    x = np.zeros((1, 64))
    x[0, :12] = [6.9, -0.25, 0.26, 0.75, 1.25, 1.26, -1.75, 2.5, 3.5, 5.0, 5.1, -0.1]   # scale 1: the largest rounds to 6
    x[0, 32:36] = [7.0, -1.0, 0.5, 0.51]                                                # 7 would round to 8: scale 2
    codes, e = decoder.quantize(x)
    assert e.tolist() == [[127, 128]]
    assert codes[0, :13].tolist() == [7, 8, 1, 2, 2, 3, 12, 4, 6, 6, 7, 8, 0]           # ties go to even codes
    assert codes[0, 32:37].tolist() == [6, 9, 0, 1, 0]
    assert decoder.values(codes, e)[0, :6].tolist() == [6, -0.0, 0.5, 1, 1, 1.5]


def test_quantize_borders():
    for v, exp in ((0.0, 0), (2.0 ** -149, 0), (6.9 * 2.0 ** -127, 0), (7 * 2.0 ** -127, 1), (1.75 * 2.0 ** 126, 252), (1.75 * 2.0 ** 127, 252), (1.99 * 2.0 ** 127, 252)):
        codes, e = decoder.quantize(np.full((32,), v))
        assert e[0] == exp, (v, e)
    for v in (np.inf, -np.inf, np.nan):
        x = np.ones(64)
        x[40] = v
        codes, e = decoder.quantize(x)
        assert e[1] == 255 and e[0] != 255 and not codes[32:].any()
        assert np.isnan(decoder.values(codes, e)[32:]).all()


def test_cache_bytes_round_trip_and_keep_the_rest():
    rng = np.random.default_rng(5)
    data = rng.integers(0, 256, (3, 2, 2, 34 * 64), dtype=np.uint8)
    before = data.copy()
    c = decoder.Cache(data, 2, 64, 64)
    table = [2, -1, 0]
    written = {}
    for pos in (0, 1, 33, 63, 64, 128 + 7, 128 + 40, 500):
        for which in (0, 1):
            x = rng.normal(size=(2, 64))
            c.write(table, pos, which, x)
            written[pos, which] = x
    for (pos, which), x in written.items():
        got = c.read(table, pos, which)
        if pos in (64, 500):
            assert got is None
            continue
        assert np.array_equal(got, decoder.values(*decoder.quantize(x)))
    assert np.array_equal(data[1], before[1])
    changed = (data != before).sum()
    assert 0 < changed <= 6 * 2 * 2 * (32 + 32 + 2)


def test_attend_is_the_library_softmax_in_64_bits():
    rng = np.random.default_rng(6)
    q, k, v = rng.normal(size=(5, 4, 32)), rng.normal(size=(9, 2, 32)), rng.normal(size=(9, 2, 32))
    vis = np.arange(9)[None, :] <= np.arange(5)[:, None] + 2
    o, _, _ = decoder.attend(q, k, v, vis, 0.3)
    for h in range(4):
        s = torch.from_numpy(q[:, h] @ k[:, h // 2].T * 0.3).masked_fill(torch.from_numpy(~vis), float("-inf"))
        assert np.allclose(o[:, h], (torch.softmax(s, -1) @ torch.from_numpy(v[:, h // 2])).numpy(), rtol=1e-12, atol=1e-14)
    assert not decoder.attend(q, k, v, np.zeros((5, 9), dtype=bool), 0.3)[0].any()


def test_rope_turns_complex_numbers():
    rng = np.random.default_rng(7)
    x, w = rng.normal(size=(6, 3, 32)), rng.normal(size=32)
    pos, freq = np.array([0, 1, 2, 1000, 1 << 20, 5]), 10000.0 ** (-np.arange(0, 24, 2) / 24)
    n = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + 1e-6) * w
    turn = np.exp(1j * pos[:, None] * freq)[:, None, :]
    half, inter = decoder.rope(x, w, 1e-6, pos, freq, 24, False), decoder.rope(x, w, 1e-6, pos, freq, 24, True)
    z = (n[..., :12] + 1j * n[..., 12:24]) * turn
    assert np.allclose(half[..., :12], z.real) and np.allclose(half[..., 12:24], z.imag) and np.allclose(half[..., 24:], n[..., 24:])
    z = (n[..., 0:24:2] + 1j * n[..., 1:24:2]) * turn
    assert np.allclose(inter[..., 0:24:2], z.real) and np.allclose(inter[..., 1:24:2], z.imag)
