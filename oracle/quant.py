"""Block-scaled 8- and 4-bit codes of K/V rows, by their definition in float64.

A row of D values is blocks of 32.  A block has a scale 2^s, s the smallest integer >= s_min with
max |x| <= M 2^s, and a code a value: the code value nearest to x 2^-s, ties to the even code, of those
whose value times 2^s does not exceed 65504, the largest float16 value.  The sign is kept, zeros included.

    8 bits: e4m3 (exponent bias 7, no infinities, code 127 is no value), M = 448, s_min = -15
    4 bits: e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6), M = 6, s_min = -23
"""

import numpy as np

BLOCK = 32
F16_MAX = 65504.0


def code_values(bits):
    """The non-negative code values in the order of their codes."""
    if bits == 4:
        return np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float64)
    out = []
    for c in range(127):
        e, m = c >> 3, c & 7
        out.append(m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return np.array(out)


def quantize(x, bits):
    """(codes uint8 [..., D], one a value with the sign in its top bit; s int [..., D / 32])."""
    x = np.asarray(x, dtype=np.float64)
    blocks = x.reshape(*x.shape[:-1], -1, BLOCK)
    grid = code_values(bits)
    amax = np.abs(blocks).max(-1)
    s = np.full(amax.shape, -15 if bits == 8 else -23)
    while (amax > grid[-1] * np.exp2(s)).any():
        s = s + (amax > grid[-1] * np.exp2(s))
    a = np.abs(blocks) / np.exp2(s)[..., None]
    up = np.searchsorted(grid, a).clip(0, len(grid) - 1)  # first code value >= a
    down = (up - 1).clip(0)
    near_up, near_down = grid[up] - a, a - grid[down]
    code = np.where(near_up < near_down, up, np.where(near_down < near_up, down, np.where(up % 2 == 0, up, down)))
    code = np.where(grid[code] * np.exp2(s)[..., None] > F16_MAX, code - 1, code)
    code = code + np.signbit(blocks) * (1 << (bits - 1))
    return code.reshape(x.shape).astype(np.uint8), s


def dequantize(codes, s, bits):
    """The values of codes [..., D] and scales s [..., D / 32], float64."""
    grid = code_values(bits)
    sign = 1 << (bits - 1)
    mag = grid[(codes & (sign - 1)).astype(np.int64)]
    v = np.where(codes & sign, -mag, mag)
    return v * np.repeat(np.exp2(s.astype(np.float64)), BLOCK, axis=-1)


def round_trip(x, bits):
    return dequantize(*quantize(x, bits), bits)


def pack(codes, bits):
    """Code bytes [..., D * bits / 8]: 4-bit codes two a byte, the even dim low."""
    return codes if bits == 8 else codes[..., ::2] | (codes[..., 1::2] << 4)


def records(K, V, k_bits, v_bits):
    """Records uint8 [..., bytes] of rows K, V [..., D]."""
    parts, scales = [], []
    for x, bits in ((K, k_bits), (V, v_bits)):
        codes, s = quantize(x, bits)
        parts.append(pack(codes, bits))
        scales.append((s + 127).astype(np.uint8))
    body = np.concatenate(parts + scales, axis=-1)
    pad = -body.shape[-1] % 16
    return np.concatenate([body, np.zeros(body.shape[:-1] + (pad,), np.uint8)], axis=-1)
