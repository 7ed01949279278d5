"""Rotations by far angles, where a rounding of the angle would show: turns against exact ones."""

from fractions import Fraction

import numpy as np
import pytest

import paper_2602_07721_amd as pk
from new_tokens import D, gpu
from pages import config, ints

pytestmark = pytest.mark.gpu

PI = Fraction("3.14159265358979323846264338327950288419716939937510582097494459")
# Positions and frequencies with angles below 2^31 near a multiple of a quarter turn, for which position * frequency /
# (2 pi) in 64 bits, rounded at each step, is off by 2^-21.2 to 2^-21.4 radians.
FAR = [(2012551875, "0x1.e634e4p-1"), (2120408143, "0x1.bb99c4p-1"), (1969003798, "0x1.d30c62p-1"),
       (2033665775, "0x1.f9c3e4p-1"), (2109541418, "0x1.99e8bep-1"), (2063542574, "0x1.ead2b2p-1"),
       (1977044310, "0x1.e1823ap-1"), (2021013805, "0x1.acd41cp-1")]


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("sign", [1, -1])
def test_far_angles_lose_whole_turns_only(pairs, sign):
    positions = [sign * p for p, _ in FAR] + [-2 ** 31, 2 ** 31 - 1, 0, 1]
    freqs = np.array([float.fromhex(f) for _, f in FAR], dtype=np.float32)
    t, half = len(positions), len(freqs)
    first, second = (2 * np.arange(half), 2 * np.arange(half) + 1) if pairs else (np.arange(half), half + np.arange(half))
    x = np.zeros((t, 1, D), np.float16)
    x[:, 0, first] = 60000
    cache = pk.PagedCache(gpu(np.zeros((1, 1, 16, D), np.float16)), gpu(np.zeros((1, 1, 16, D), np.float16)))
    got = pk.rotate_rows(config(1, 1), cache, gpu(x), gpu(x), gpu(x), ints(positions), ints(np.arange(t)), gpu(freqs),
                         pairs=pairs).cpu().numpy().astype(np.float64)[:, 0]
    keys = cache.K[0, 0, :t].cpu().numpy().astype(np.float64)
    turns = np.empty((t, half))
    for i, p in enumerate(positions):
        for j, f in enumerate(freqs):
            turn = Fraction(p) * Fraction(float(f)) / (2 * PI)
            turns[i, j] = float(turn - round(turn))
    for at, want in ((first, np.cos(2 * np.pi * turns)), (second, np.sin(2 * np.pi * turns))):
        # Of 60000: the sine's or cosine's 2^-22.9, the turns' rounding to float32 (2^-26 of a turn) and that of the
        # product; half a float16 step of the output.
        tol = 60000 * (2.0 ** -22.9 + 2 * np.pi * 2.0 ** -26 + 2.0 ** -24) + 60000 * np.abs(want) * 2.0 ** -11
        for y in (got, keys):
            off = np.abs(y[:, at] - 60000 * want) / tol
            assert (off <= 1).all(), f"off by {off.max():.3g} of what is allowed"


# Angles next to whole turns, for which what position * frequency and 1 / (2 pi) lose in 64 bits is 2^-21.9 radians.
WHOLE = [(2144616710, "0x1.fe90aap-1"), (2147390953, "0x1.fc44acp-1"), (2138889594, "0x1.fdf17ep-1"),
         (2145705929, "0x1.fbf2acp-1"), (2130319918, "0x1.ff56aap-1"), (2144759454, "0x1.fb773ap-1"),
         (2146530601, "0x1.fae1fcp-1"), (2132785550, "0x1.fdf2e2p-1")]


@pytest.mark.parametrize("pairs", [False, True])
def test_angles_next_to_whole_turns_are_their_small_parts(pairs):
    # Token i turns pair i by its far angle, or, as token 0 of position 1, by what is left of it, in float32.  The two
    # angles differ by 2^-24 of one below 2^-14, so the sines by next to nothing: allowed are half a float16 step of
    # either output and 2^-24 of 60000 for the products.
    half = len(WHOLE)
    freqs = np.array([float.fromhex(f) for _, f in WHOLE], dtype=np.float32)
    left = []
    for p, f in WHOLE:
        turn = Fraction(p) * Fraction(float.fromhex(f)) / (2 * PI)
        left.append(float((turn - round(turn)) * 2 * PI))
    assert max(abs(x) for x in left) < 2.0 ** -14
    x = np.zeros((half, 1, D), np.float16)
    first, second = (2 * np.arange(half), 2 * np.arange(half) + 1) if pairs else (np.arange(half), half + np.arange(half))
    x[:, 0, first] = 60000

    def sines(positions, freqs):
        cache = pk.PagedCache(gpu(np.zeros((1, 1, 16, D), np.float16)), gpu(np.zeros((1, 1, 16, D), np.float16)))
        return pk.rotate_rows(config(1, 1), cache, gpu(x), gpu(x), gpu(x), ints(positions), ints(np.arange(half)), gpu(freqs),
                              pairs=pairs).cpu().numpy().astype(np.float64)[:, 0, second]

    far = np.diag(sines([p for p, _ in WHOLE], freqs))
    near = sines([1] * half, np.array(left, np.float32))[0]
    off = np.abs(far - near) / (np.abs(near) * 2.0 ** -10 + 60000 * 2.0 ** -24)
    assert (off <= 1).all(), f"off by {off} of what is allowed"
