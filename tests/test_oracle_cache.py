"""Pins of the quantised cache's oracle: the formats, the choice of a scale, rounding, and
rotations along several axes.  CPU only."""
import numpy as np
import pytest
import torch

from oracle import cache as oc


def test_grids_are_the_formats():
    assert list(oc.E2M1) == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    want = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(oc.E4M3, want)


def test_eight_bit_codes_are_torch_s():
    x = torch.randn(50, 64, generator=torch.Generator().manual_seed(0)) * 100
    x[0] = 448 * torch.sign(x[0])
    x = x.clamp(-448, 448)
    x[:, 0] = x[:, 32] = 448                    # so that every group's scale is 1
    codes, scales = oc.quantise(x.numpy(), 8)
    assert (scales == 127).all()
    assert np.array_equal(codes, x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())


@pytest.mark.parametrize("bits", [4, 8])
def test_scale_is_the_least_that_holds_the_group(bits):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((300, 32)) * 2.0 ** rng.integers(-100, 100, size=(300, 1))
    top = np.abs(x).max(-1)
    last = oc.GRID[bits][-1]
    x[:50, 0] = last * 2.0 ** np.floor(np.log2(top[:50]))       # exactly at the end
    top = np.abs(x).max(-1)
    _, scales = oc.quantise(x, bits)
    e = scales[:, 0].astype(int) - 127
    assert (top <= last * 2.0 ** e).all() and (top > last * 2.0 ** (e - 1)).all()


@pytest.mark.parametrize("bits", [4, 8])
def test_nearest_value_and_ties_to_even(bits):
    grid = oc.GRID[bits]
    mid = (grid[1:] + grid[:-1]) / 2
    x = np.zeros((len(mid), 32))
    x[:, 0], x[:, 1], x[:, 2] = grid[-1], mid, -mid
    x[:, 3], x[:, 4] = np.nextafter(mid, 1e9), np.nextafter(mid, 0)
    codes, scales = oc.quantise(x, bits)
    assert (scales == 127).all()
    half = 8 if bits == 4 else 128
    even = np.arange(len(mid)) + np.arange(len(mid)) % 2
    assert np.array_equal(codes[:, 1], even) and np.array_equal(codes[:, 2], even + half)
    assert np.array_equal(codes[:, 3], np.arange(len(mid)) + 1)
    assert np.array_equal(codes[:, 4], np.arange(len(mid)))
    # values: nothing nearer
    v = oc.values(codes, scales, bits)
    both = np.concatenate([-grid[::-1], grid])
    assert np.array_equal(np.abs(v - x), np.abs(x[..., None] - both).min(-1))


@pytest.mark.parametrize("bits", [4, 8])
def test_values_of_codes_and_their_bytes(bits):
    codes = np.arange(16 if bits == 4 else 256, dtype=np.uint8)
    codes = np.resize(codes, (8, 64))
    data = oc.pack_codes(codes, bits)
    assert data.shape == (8, 64 * bits // 8)
    assert np.array_equal(oc.unpack_codes(data, bits), codes)
    if bits == 4:
        assert data[0, 0] == 0x10 and data[0, 7] == 0xfe     # element 2i in the low half
    s = np.full((8, 2), 127, dtype=np.uint8)
    one = oc.values(codes, s, bits)
    s[1], s[2] = (126, 130), (255, 127)
    v = oc.values(codes, s, bits)
    assert np.array_equal(v[1, :32], one[1, :32] / 2, equal_nan=True)
    assert np.array_equal(v[1, 32:], one[1, 32:] * 8, equal_nan=True)
    assert np.isnan(v[2, :32]).all() and np.array_equal(v[2, 32:], one[2, 32:], equal_nan=True)


@pytest.mark.parametrize("bits", [4, 8])
def test_ends_of_the_range(bits):
    x = np.zeros((4, 32))
    x[0, 0], x[1, 0], x[2, 0], x[3, 5] = np.finfo(np.float32).max, 2.0 ** -140, np.nan, -np.inf
    codes, scales = oc.quantise(x, bits)
    lo, hi = oc.EXPONENTS[bits]
    assert list(scales[:, 0]) == [hi + 127, lo + 127, 255, 255]
    v = oc.values(codes, scales, bits)
    assert np.isfinite(v[0]).all() and v[0, 0] == oc.GRID[bits][-1] * 2.0 ** hi and v[1, 0] == 0


def test_rotation_keeps_norms_and_depends_on_differences():
    rng = np.random.default_rng(0)
    d, axis = 64, [0, 1, 2] * 8
    freq = [50.0 ** (-j / 24) for j in range(24)]
    q, k = rng.standard_normal((2, 5, 1, d))
    p, m = rng.integers(-50, 50, size=(2, 3, 5))
    shift = np.array([[3], [-8], [21]])
    for pairing in ("halves", "neighbours"):
        def turn(x, pos):
            return oc.rotary_axes(x, pos, freq, axis, pairing)
        a = (turn(q, p) * turn(k, m)).sum(-1)
        assert np.allclose(a, (turn(q, p + shift) * turn(k, m + shift)).sum(-1))
        assert not np.allclose(a, (turn(q, p + shift) * turn(k, m)).sum(-1))
        assert np.allclose((turn(q, p) ** 2).sum(-1), (q ** 2).sum(-1))
        assert np.array_equal(turn(q, p)[..., 48:], q[..., 48:])
        assert np.array_equal(turn(q, 0 * p), q)
    # a pair as a complex number, by hand
    x = np.zeros((1, 1, 4))
    x[0, 0] = 1, 2, 3, 4
    y = oc.rotary_axes(x, np.array([[2], [5]]), [0.1, 0.3], [1, 0], "halves")[0, 0]
    z = [(1 + 3j) * np.exp(0.5j), (2 + 4j) * np.exp(0.6j)]
    assert np.allclose(y, [z[0].real, z[1].real, z[0].imag, z[1].imag])
    y = oc.rotary_axes(x, np.array([[2], [5]]), [0.1, 0.3], [1, 0], "neighbours")[0, 0]
    z = [(1 + 2j) * np.exp(0.5j), (3 + 4j) * np.exp(0.6j)]
    assert np.allclose(y, [z[0].real, z[0].imag, z[1].real, z[1].imag])


def test_attention_by_hand_and_without_scale():
    rng = np.random.default_rng(2)
    k, v = rng.standard_normal((2, 9, 2, 8))
    q = rng.standard_normal((3, 4, 8))
    out = oc.attention(q, k, v, [1, 9, 4], 0.3)
    assert np.allclose(out[0], v[0].repeat(2, axis=0))           # one key: its value
    z = 0.3 * k[:4, 1] @ q[2, 3]
    assert np.allclose(out[2, 3], (np.exp(z) / np.exp(z).sum()) @ v[:4, 1])
    assert np.allclose(oc.attention(0 * q, k, v, [9] * 3, 1.0)[1, 0], v[:, 0].mean(0))
