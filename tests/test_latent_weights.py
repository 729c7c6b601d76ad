"""The weights of the absorbed form in plain numpy: terms of four bits each, every term sixteen times finer than the one before,
counted from the largest weight of 64 tokens.

A term is a value of e4m3 rounded to nearest, off by at most 2^-4 for y in [1, 2).  That rest times 16 is at most 1, of which the second
term is off by at most 2^-5: 2^-9 of the weight; what is left times 256 is at most 2^-1, of which the third is off by at most
2^-6: 2^-14.  So it is for every y for which such a last term is a normal number, 2^-6 or more: y of 2^-5 or more (two terms; 2^-4 for three).  Below, the
last term's half step is 2^-10, 2^-14 or 2^-18 of y's unit.  The largest y is in [2^7, 2^8).
"""
import numpy as np
import pytest

from oracle.kv import decode, encode

TERMS = {"bf16": 2, "fp16": 3}
BITS = {1: 2.0 ** -4, 2: 2.0 ** -9, 3: 2.0 ** -14}


def split(y, terms):
    """What y enters the product as."""
    out, rest = np.zeros_like(y), y
    for k in range(terms):
        part = decode(encode(rest, "e4m3fn"), "e4m3fn")
        out = out + part * 2.0 ** (-4 * k)
        rest = (rest - part) * 16
    return out


def weights(g, terms, frame):
    """2^g as the product has it; `frame`: tokens that share a largest weight."""
    out = np.empty_like(g)
    for i in range(0, len(g), frame):
        top = np.floor(g[i:i + frame].max())
        out[i:i + frame] = split(2.0 ** (g[i:i + frame] - top + 7), terms) * 2.0 ** (top - 7)
    return out


@pytest.mark.parametrize("terms", [1, 2, 3])
def test_a_weight_has_its_bits(terms):
    y = 2.0 ** np.linspace({1: -6, 2: -5, 3: -4}[terms], 8, 20001)
    off = np.abs(split(y, terms) - y) / y
    assert (off <= BITS[terms]).all() and off.max() > BITS[terms] / 2      # and no fewer terms would do
    least = 2.0 ** np.linspace(-40, -6, 4001)
    assert (np.abs(split(least, terms) - least) <= 2.0 ** -10 * 16.0 ** (1 - terms)).all()


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("tokens,share", [(8190, 0.5), (8190, 0.9), (16383, 0.7), (60000, 0.5), (60000, 0.9)])
def test_many_small_weights_beside_a_large_one(kind, tokens, share):
    """The sum of the small ones, which all point one way.  Counted from the largest of 64 each keeps its bits but for the
    63 beside the large one; counted from the largest of all, those below half a step would be gone."""
    g = np.random.default_rng(0)
    tail = (1 - share) / share / (tokens - 1)
    x = np.log2(tail) + g.standard_normal(tokens) * 0.3
    x[0] = 0
    exact, terms = 2.0 ** x, TERMS[kind]
    tol = BITS[terms] * exact[1:].sum() + 63 * 2.0 ** -17 * 16.0 ** (1 - terms)
    assert abs(weights(x, terms, 64)[1:].sum() - exact[1:].sum()) <= tol
    assert tol < 0.01 * exact[1:].sum()
    if kind == "bf16" and tail < 2.0 ** -18:                              # with 2^3 as the largest of all
        assert split(2.0 ** (x + 3), terms)[1:].sum() < exact[1:].sum()


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_one_term_less_is_seen(kind):
    """Of weights that are alike all are off alike: 32 fractions of an octave, as the GPU's test has them."""
    least = [np.abs(split(2.0 ** (7 + np.arange(32) / 32), TERMS[kind] - less) / 2.0 ** (7 + np.arange(32) / 32) - 1).max() for less in (0, 1)]
    out = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}[kind]                    # a value's own rounding
    assert least[0] <= BITS[TERMS[kind]] and least[1] > 1.5 * (out + BITS[TERMS[kind]])
