"""GPU: sines and cosines of rotary positions, place by place.

With x the rest of the angle after whole quarter turns, |x| <= pi / 4, in halves of the step 2^-24 that numbers of 1/2 to 1 have, 2^-25:
sine x + t, |t| < 0.09: the sum's rounding (1), t's products' (0.09 * 2^-24 each, three of them: 0.5), the series (0.07);
cosine 1 + u, |u| < 0.3: the sum's rounding (1), that of x x, halved (0.5), u's factor's (0.4) and its own (0.5), the series (0.01).
The angle: 2^-51 of it.  Before a rest's own rounding was made good it was off by 1 more, times the other function's 0.7 to 1.
"""
import numpy as np
import pytest
import torch

from test_gpu_rotary import dev, ints, np_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def uz():
    import paper_2604_17172_amd as m
    return m


@pytest.mark.parametrize("interleaved", [False, True])
def test_sines_and_cosines(uz, interleaved):
    g = np.random.default_rng(3)
    rows, half = 20000, 16
    places, freq = np.arange(-rows // 2, rows // 2), g.uniform(0.01, 1.0, half).astype(np.float32)
    x = torch.zeros(rows, 1, 2 * half, device="cuda")
    x[..., slice(0, None, 2) if interleaved else slice(0, half)] = 1      # (1, 0) turned is (cosine, sine)
    got = np_of(uz.rotate(x, ints(places), dev(freq), interleaved=interleaved))[:, 0]
    c, s = (got[:, 0::2], got[:, 1::2]) if interleaved else (got[:, :half], got[:, half:])
    angle = places[:, None].astype(np.float64) * freq
    quarter = np.rint(angle / (np.pi / 2)).astype(np.int64) & 1            # of odd ones the sine's series makes the cosine
    for value, want, by_sine in ((c, np.cos(angle), quarter == 1), (s, np.sin(angle), quarter == 0)):
        off = np.abs(value - want) - 2.0 ** -50 * np.abs(angle)
        assert (off[by_sine] <= 1.6 * 2.0 ** -25).all(), off[by_sine].max() * 2.0 ** 25
        assert (off[~by_sine] <= 2.45 * 2.0 ** -25).all(), off[~by_sine].max() * 2.0 ** 25


def test_cosines_within_a_step(uz):
    """1 - x x / 2 with what its product and its sum leave, and a tail |u| < 0.016: the last sum's rounding (1), the tail's (0.2), the
    series (0.01)."""
    places = np.arange(-(1 << 18), 1 << 18)
    freq = np.array([2.0 ** -12 * np.pi / 8], np.float32)               
    x = torch.zeros(len(places), 1, 2, device="cuda")
    x[..., 0] = 1
    got = np_of(uz.rotate(x, ints(places), dev(freq)))[:, 0]
    angle = places.astype(np.float64) * freq.astype(np.float64)
    odd = np.rint(angle / (np.pi / 2)).astype(np.int64) & 1
    value, want = np.where(odd, got[:, 1], got[:, 0]), np.where(odd, np.sin(angle), np.cos(angle))
    off = np.abs(value - want) - 2.0 ** -50 * np.abs(angle)
    assert (off <= 1.25 * 2.0 ** -25).all(), off.max() * 2.0 ** 25


@pytest.mark.parametrize("magnitude", [1.2, 0.1 * np.log(7) + 1, 1 / 3, -1.1])
def test_magnitudes_that_32_bits_do_not_hold(uz, magnitude):
    """m (1, 0) turned: beside the functions' own errors, at most 1.6 and 1.25 half steps of 1/2 to 1 times m, the product's rounding."""
    places, freq = np.arange(40000), np.array([0.37, 1.0, 0.001], np.float32)
    x = torch.zeros(len(places), 1, 6, device="cuda")
    x[..., :3] = 1
    got = np_of(uz.rotate(x, ints(places), dev(freq), magnitude=magnitude))[:, 0]
    angle = places[:, None].astype(np.float64) * freq
    want = magnitude * np.concatenate([np.cos(angle), np.sin(angle)], axis=1)
    tail = np.where(np.abs(want) <= abs(magnitude) * 0.7072, 0.6, 0.25)   # what a function is off by beside its last rounding, which is the product's
    step = 2.0 ** (np.floor(np.log2(np.abs(want) + 2.0 ** -60)) - 23)
    tol = step / 2 + (tail * 2.0 ** -25 + 2.0 ** -50 * np.tile(angle, 2)) * abs(magnitude) * (1 + 2.0 ** -20)
    assert (np.abs(got - want) <= tol).all(), (np.abs(got - want) / tol).max()


def test_turns_are_refused_by_their_magnitude_in_32_bits(uz):
    x, places, freq = torch.zeros(1, 1, 2, device="cuda"), ints([0]), dev(np.ones(1, np.float32))
    for magnitude in (1e39, -1e39, float("inf"), float("nan")):
        with pytest.raises(uz.UzipError):
            uz.rotate(x, places, freq, magnitude=magnitude)
