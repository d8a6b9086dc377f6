"""The oracle of a pool held in 4 or 8 bits: pinned to exact rational arithmetic, to the layout
element by element, and to mistakes planted in it."""

from fractions import Fraction

import numpy as np
import pytest

import oracle.quant_cache as qc
from oracle import bf16_bits_to_f64, pack_tiles, quantise_rows, row_values, split_tiles, to_bf16_bits, unpack_tiles
from quant_util import spread_rows

FORMATS = [4, 8]


def numbers_of(nbits):
    """The format's numbers by its definition, sign aside, as fractions by code."""
    exp_bits, man_bits, bias = {4: (2, 1, 1), 8: (4, 3, 7)}[nbits]
    out = []
    for code in range(1 << (nbits - 1)):
        e, m = code >> man_bits, code & ((1 << man_bits) - 1)
        if nbits == 8 and code == 127:
            continue
        if e == 0:
            out.append(Fraction(m, 1 << man_bits) * Fraction(2) ** (1 - bias))
        else:
            out.append((1 + Fraction(m, 1 << man_bits)) * Fraction(2) ** (e - bias))
    assert len(out) == (8 if nbits == 4 else 127) and exp_bits + man_bits + 1 == nbits
    return out


def nearest(x, numbers):
    """Code of the nearest number to the fraction x >= 0, ties to the even code."""
    d = [abs(x - n) for n in numbers]
    best = min(d)
    codes = [c for c, v in enumerate(d) if v == best]
    return codes[0] if len(codes) == 1 else next(c for c in codes if c % 2 == 0)


def smallest_exponent(most, nbits):
    """By the definition: no rounding beyond the largest number, were there one more."""
    numbers = numbers_of(nbits)
    further = numbers + [{4: Fraction(8), 8: Fraction(480)}[nbits]]
    lo, hi = {4: (-125, 125), 8: (-117, 119)}[nbits]
    for e in range(lo, hi + 1):
        x = most / Fraction(2) ** e
        if x <= further[-1] and nearest(x, further) < len(numbers):
            return e
    return hi


@pytest.mark.parametrize("nbits", FORMATS)
def test_numbers(nbits):
    assert [Fraction(x) for x in qc.NUMBERS[nbits]] == numbers_of(nbits)
    assert max(numbers_of(nbits)) == {4: 6, 8: 448}[nbits]


@pytest.mark.parametrize("nbits", FORMATS)
def test_rows_against_rational_arithmetic(nbits):
    rng = np.random.default_rng(1)
    rows = [spread_rows(rng, 6, 32)]
    # borders and their neighbours, the ends of the exponent's range, subnormal numbers
    edge = np.zeros((8, 32), dtype=np.uint16)
    edge[0, :6] = [0x40DF, 0x40E0, 0x40E1, 0x3E80, 0x3E7F, 0xC0A0]      # about 7, .25, 5
    edge[1, :4] = [0x43E8, 0x43E9, 0x43E7, 0x3A80]                       # 464, 466, 462, 2^-10
    edge[2, :3] = [0x7F7F, 0xFF7F, 0x7F00]
    edge[3, :4] = [0x7F68, 0x7F60, 0x7F40, 0x0080]
    edge[4, :4] = [0x0001, 0x007F, 0x8001, 0x0000]
    edge[5, :3] = [0x0100, 0x0180, 0x0090]
    edge[6, :3] = [0x05C0, 0x0380, 0x8000]
    rows = np.concatenate(rows + [edge])
    codes, scales = quantise_rows(rows, nbits)
    numbers = numbers_of(nbits)
    for row, c, s in zip(rows, codes, scales):
        x = [Fraction(float(v)) for v in bf16_bits_to_f64(row)]
        e = smallest_exponent(max(abs(v) for v in x), nbits)
        assert s[0] == e + 127
        for v, bits, code in zip(x, row, c):
            want = nearest(min(abs(v) / Fraction(2) ** e, numbers[-1]), numbers)
            assert code == want | (int(bits) >> 15) << (nbits - 1)
    values = row_values(codes, scales, nbits)
    to_bf16_bits(values)                                    # every value is a bf16 number
    assert np.isfinite(values).all()


@pytest.mark.parametrize("nbits", FORMATS)
def test_values_are_within_half_a_step(nbits):
    """Relative to a feature at most eps / 2 of the format, or half a subnormal step."""
    rng = np.random.default_rng(2)
    rows = spread_rows(rng, 50, 128)
    codes, scales = quantise_rows(rows, nbits)
    x, y = bf16_bits_to_f64(rows), row_values(codes, scales, nbits)
    step = np.exp2(scales.astype(float) - 127).repeat(32, -1) * {4: 0.25, 8: 2.0 ** -10}[nbits]
    assert (np.abs(x - y) <= np.maximum(np.abs(x) * {4: 2.0 ** -2, 8: 2.0 ** -4}[nbits], step)).all()


@pytest.mark.parametrize("nbits", FORMATS)
def test_what_is_not_finite_makes_its_group_nan(nbits):
    rows = np.zeros((3, 64), dtype=np.uint16)
    rows[:] = 0x3F80
    rows[0, 3], rows[1, 40], rows[2, 63] = 0x7FC0, 0x7F80, 0xFF80
    y = row_values(*quantise_rows(rows, nbits), nbits)
    assert (np.isnan(y) == [[True] * 32 + [False] * 32, [False] * 32 + [True] * 32, [False] * 32 + [True] * 32]).all()


@pytest.mark.parametrize("nbits", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
def test_layout_element_by_element(nbits, d):
    rng = np.random.default_rng(3)
    k, v = spread_rows(rng, 2, 3, 16, d), spread_rows(rng, 2, 3, 16, d)
    tiles = pack_tiles(k, v, nbits)
    assert tiles.shape == (2, 3, d * nbits * 4 + d)
    n = 16 * d * nbits // 8
    (kc, ks), (vc, vs) = quantise_rows(k, nbits), quantise_rows(v, nbits)

    def code(tile, base, i):
        return tile[base + i] if nbits == 8 else tile[base + i // 2] >> 4 * (i % 2) & 15

    for b, h in [(0, 0), (1, 2)]:
        for t in range(16):
            for f in range(d):
                assert code(tiles[b, h], 0, t * d + f) == kc[b, h, t, f]
                part = d // 16
                assert code(tiles[b, h], n, (f // part * 16 + t) * part + f % part) == vc[b, h, t, f]
            for i in range(d // 32):
                assert tiles[b, h, 2 * n + t * (d // 32) + i] == ks[b, h, t, i]
                assert tiles[b, h, 2 * n + 16 * (d // 32) + i * 16 + t] == vs[b, h, t, i]
    for got, want in zip(split_tiles(tiles, d, nbits), (kc, ks, vc, vs)):
        assert (got == want).all()
    for got, want in zip(unpack_tiles(tiles, d, nbits), (row_values(kc, ks, nbits), row_values(vc, vs, nbits))):
        assert (got == want).all()


@pytest.mark.parametrize("nbits", FORMATS)
@pytest.mark.parametrize("mistake", ["floor", "no_step_up", "ties_up", "other_group"])
def test_planted_mistakes_are_seen(nbits, mistake):
    """Each changes some value of ordinary rows: what the comparisons of values rest on."""
    rng = np.random.default_rng(4)
    rows = spread_rows(rng, 200, 64)
    codes, scales = quantise_rows(rows, nbits)
    good = row_values(codes, scales, nbits)
    x = bf16_bits_to_f64(rows).reshape(200, 2, 32)
    e = scales.astype(int) - 127
    if mistake == "no_step_up":
        e = np.frexp(np.abs(x).max(-1))[1] - 1 - qc.TOP[nbits]
    if mistake == "other_group":
        e = e[:, ::-1]
    y = np.abs(x) / np.exp2(e)[..., None]
    numbers = qc.NUMBERS[nbits]
    borders = numbers[1:] if mistake == "floor" else (numbers[1:] + numbers[:-1]) / 2
    bad = numbers[np.searchsorted(borders, y, side="right" if mistake in ("floor", "ties_up") else "left")]
    bad = np.copysign(bad * np.exp2(e)[..., None], x).reshape(rows.shape)
    assert (bad != good).any()
