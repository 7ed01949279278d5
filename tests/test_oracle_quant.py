"""Pins of the block-scaled code oracle (CPU)."""

import numpy as np
import pytest

from oracle import quant


@pytest.mark.parametrize("bits,top,last", [(8, 448.0, 126), (4, 6.0, 7)])
def test_code_values(bits, top, last):
    v = quant.code_values(bits)
    assert v[0] == 0 and v[-1] == top and len(v) == last + 1 and (np.diff(v) > 0).all()


@pytest.mark.parametrize("bits", [8, 4])
def test_nearest_code_by_brute_force(bits):
    r = np.random.default_rng(bits)
    x = (r.standard_normal((200, 32)) * np.exp2(r.integers(-24, 14, (200, 1)))).astype(np.float16).astype(np.float64)
    codes, s = quant.quantize(x, bits)
    back = quant.dequantize(codes, s, bits)
    grid = quant.code_values(bits)
    M, s_min = (448, -15) if bits == 8 else (6, -23)
    for row in range(200):
        amax, e = np.abs(x[row]).max(), int(s[row, 0])
        assert amax <= M * 2.0 ** e and (e == s_min or amax > M * 2.0 ** (e - 1))
        all_values = np.concatenate([grid, -grid]) * 2.0 ** e
        best = np.abs(all_values[None, :] - x[row][:, None]).min(1)
        assert (np.abs(back[row] - x[row]) == best).all()


@pytest.mark.parametrize("bits", [8, 4])
def test_every_stored_value_is_float16_and_kept(bits):
    r = np.random.default_rng(7)
    raw = r.integers(0, 1 << 16, (500, 128)).astype(np.uint16).view(np.float16)
    x = np.where(np.isfinite(raw), raw, np.float16(0)).astype(np.float64)
    x[0], x[1, :32], x[2, 5], x[3] = 0, 65504, -65504, 2.0 ** -24
    y = quant.round_trip(x, bits)
    assert (y == y.astype(np.float16).astype(np.float64)).all() and np.abs(y).max() <= 65504
    assert (quant.round_trip(y, bits) == y).all() and (y[3] == 2.0 ** -24).all() and (y[0] == 0).all()


@pytest.mark.parametrize("bits,x,want", [
    (8, [448, 464 - 17, 17, 18, 0.0009765625, -0.0009765625], [448, 448, 16, 18, 0, 0]),
    (4, [6, 5, 2.5, 3.5, 0.25, -0.75], [6, 4, 2, 4, 0, -1]),
    (8, [65504, 63488, 61440, 240, -65504, 8], [61440, 61440, 61440, 240, -61440, 8]),
    (4, [65504, 40960, 49152, 8192, -65504, 4096], [49152, 32768, 49152, 8192, -49152, 0])])
def test_ties_and_limits(bits, x, want):
    row = np.zeros(32)
    row[:6] = x
    assert quant.round_trip(row, bits)[:6].tolist() == want


@pytest.mark.parametrize("kb,vb,size", [(8, 8, 272), (8, 4, 208), (4, 8, 208), (4, 4, 144)])
def test_record_layout(kb, vb, size):
    K, V = np.zeros((1, 128)), np.zeros((1, 128))
    K[0, :4], V[0, 96:100] = [1, -2, 3, 0.5], [4, 4, -4, 2]
    rec = quant.records(K, V, kb, vb)[0]
    nk, nv = 16 * kb, 16 * vb
    assert rec.size == size and not rec[nk + nv + 8:].any()
    if kb == 4:  # s = 0 - 1: 3 <= 6 * 2^-1; codes of 2, -4, 6, 1
        assert rec[:2].tolist() == [4 | 14 << 4, 7 | 2 << 4] and rec[nk + nv] == 126
    else:        # s = 1 - 8: codes of 128, -256, 384, 64
        assert rec[:4].tolist() == [0x70, 0xf8, 0x7c, 0x68] and rec[nk + nv] == 120
    if vb == 4:  # s = 0: codes of 4, 4, -4, 2
        assert rec[nk + 48:nk + 50].tolist() == [6 | 6 << 4, 14 | 4 << 4] and rec[nk + nv + 7] == 127
    else:        # s = 2 - 8: codes of 256, 256, -256, 128
        assert rec[nk + 96:nk + 100].tolist() == [0x78, 0x78, 0xf8, 0x70] and rec[nk + nv + 7] == 121
    assert rec[nk + nv + 1] == (112 if kb == 8 else 104)  # an empty block: s_min
