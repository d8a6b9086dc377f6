"""Oracle of a KV pool held in 4 or 8 bits (test infrastructure).

The 32 features of a group share a scale ``2^e``; each becomes the nearest number of the
format times that, ties to the even code.  ``e`` is the smallest exponent (within the
format's bounds) for which the group's largest magnitude does not round beyond the largest
number.  Everything is evaluated in float64, where all of it is exact.
"""

import numpy as np

from .paged_attention import bf16_bits_to_f64

GROUP = 32
BLOCK = 16
NAN_BYTE = 255

# the numbers from 0 up, in the order of their codes
NUMBERS = {
    4: np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6]),
    8: np.array([m * 2.0 ** -9 for m in range(8)]
                + [(8 + m) * 2.0 ** (e - 3) for e in range(-6, 9) for m in range(8)][:-1]),
}
# exponent of the largest number, and the bounds of e
TOP = {4: 2, 8: 8}
BOUNDS = {4: (-125, 125), 8: (-117, 119)}


def _rounds_beyond(x, nbits):
    """Whether magnitude x (relative to the scale) is nearer to the number that would follow the
    largest one: 8 after 6 (7 goes there, 6 has an odd code), 480 after 448 (464 does not)."""
    return x >= 7 if nbits == 4 else x > 464


def quantise_rows(bits, nbits):
    """Codes (uint8, shape of ``bits``) and scale bytes (uint8, one per 32 features) of bf16 rows."""
    x = bf16_bits_to_f64(bits)
    g = x.reshape(*x.shape[:-1], -1, GROUP)
    most = np.abs(g).max(-1)
    bad = ~np.isfinite(g).all(-1)
    most = np.where(bad, 1.0, most)
    lo, hi = BOUNDS[nbits]
    e = np.where(most > 0, np.frexp(most)[1] - 1 - TOP[nbits], lo)
    e = e + np.where(_rounds_beyond(most / np.exp2(e), nbits), 1, 0)
    e = np.clip(e, lo, hi)
    y = np.where(bad[..., None], 0.0, g) / np.exp2(e)[..., None]
    numbers = NUMBERS[nbits]
    borders = (numbers[1:] + numbers[:-1]) / 2
    code = np.searchsorted(borders, np.abs(y), side="left")         # at a border: the lower one
    tie = (code < len(borders)) & (np.abs(y) == borders[np.minimum(code, len(borders) - 1)])
    code = code + (tie & (code % 2 == 1))
    code = code | np.where(np.signbit(y), 1 << (nbits - 1), 0)
    return (code.reshape(x.shape).astype(np.uint8), np.where(bad, NAN_BYTE, e + 127).astype(np.uint8))


def row_values(codes, scales, nbits):
    """What codes and scale bytes stand for, in float64."""
    numbers = NUMBERS[nbits]
    if nbits == 8:
        numbers = np.append(numbers, np.nan)
    x = np.concatenate([numbers, -numbers])[codes]
    x = x.reshape(*codes.shape[:-1], -1, GROUP)
    scale = np.where(scales == NAN_BYTE, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return (x * scale[..., None]).reshape(codes.shape)


def _halves(codes, nbits):
    return codes if nbits == 8 else codes[..., 0::2] | codes[..., 1::2] << 4


def _codes(data, nbits):
    return data if nbits == 8 else np.stack([data & 15, data >> 4], -1).reshape(*data.shape[:-1], -1)


def pack_tiles(k_bits, v_bits, nbits):
    """The tiles ``[blocks, KV heads, bytes]`` of bf16 blocks ``[blocks, KV heads, 16, D]``."""
    nb, h, _, d = k_bits.shape
    kc, ks = quantise_rows(k_bits, nbits)
    vc, vs = quantise_rows(v_bits, nbits)
    vc = vc.reshape(nb, h, BLOCK, 16, d // 16).swapaxes(2, 3)
    parts = [_halves(kc.reshape(nb, h, -1), nbits), _halves(vc.reshape(nb, h, -1), nbits),
             ks.reshape(nb, h, -1), vs.swapaxes(2, 3).reshape(nb, h, -1)]
    return np.ascontiguousarray(np.concatenate(parts, 2))


def split_tiles(tiles, d, nbits):
    """Codes and scale bytes of K and V as ``[blocks, KV heads, 16, ...]``: kc, ks, vc, vs."""
    nb, h, _ = tiles.shape
    n, g = BLOCK * d * nbits // 8, BLOCK * d // GROUP
    kc = _codes(tiles[:, :, :n], nbits).reshape(nb, h, BLOCK, d)
    vc = _codes(tiles[:, :, n:2 * n], nbits).reshape(nb, h, 16, BLOCK, d // 16).swapaxes(2, 3)
    ks = tiles[:, :, 2 * n:2 * n + g].reshape(nb, h, BLOCK, -1)
    vs = tiles[:, :, 2 * n + g:].reshape(nb, h, -1, BLOCK).swapaxes(2, 3)
    return kc, ks, vc.reshape(nb, h, BLOCK, d), vs


def unpack_tiles(tiles, d, nbits):
    """K and V of the tiles in float64, ``[blocks, KV heads, 16, D]``."""
    kc, ks, vc, vs = split_tiles(tiles, d, nbits)
    return row_values(kc, ks, nbits), row_values(vc, vs, nbits)


def to_bf16_bits(x):
    """Bits of float64 values that are bf16 numbers (asserted); NaN as 0x7FC0."""
    with np.errstate(over="ignore"):
        w = x.astype(np.float32).view(np.uint32)
    bits = np.where(np.isnan(x), 0x7FC0, w >> 16).astype(np.uint16)
    assert (np.isnan(x) | (bf16_bits_to_f64(bits) == x)).all(), "not a bf16 number"
    return bits
