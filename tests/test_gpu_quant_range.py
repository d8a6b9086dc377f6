"""Attention over a pool held in 4 or 8 bits at the ends of the numbers' range: values near the
format's largest and far below 1."""

import numpy as np
import pytest

from bounded_cache_util import bf16_bits
from oracle import window_attention
from quant_util import QuantPaged, quant_attention_bound
from test_gpu_quant_attention import run_decode, run_prefill

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

HQ, HKV = 8, 2


def scaled(bits, power):
    """bf16 bits of numbers times 2^power, exactly; zeros and NaN as they are."""
    x = bits.copy()
    x[((bits & 0x7F80) != 0) & ((bits & 0x7F80) != 0x7F80)] += np.uint16(power << 7 & 0xFFFF)
    return x


def compare(got, q, pg, r, first, d, unit=1.0):
    """Rows at positions first .. of sequence r, outputs and bound in units of `unit`."""
    scale = float(np.float32(d ** -0.5))
    out, mag = window_attention(q, pg.k, pg.v, pg.tables[r], first, HQ, HKV, scale)
    got, out, mag = got / unit, out / unit, mag / unit
    assert np.isfinite(got).all(), f"sequence {r}: {(~np.isfinite(got)).sum()} elements are not finite"
    err = np.abs(got - out)
    assert (err <= quant_attention_bound(out, mag)).all(), f"sequence {r}: {err.max()}"


# (prefix, suffix) of a launch in key parts and of one that fills the device's work-groups
INVOCATIONS = {"parts": [(1000, 21), (0, 40)], "whole": [(60, 700)] * 14}


def both(pg, q, qp, invs, bits, d, unit=1.0):
    """Decode of the sequences' last tokens and prefill of their suffixes."""
    scale = float(np.float32(d ** -0.5))
    got = run_decode(pg, q, bits, scale)
    for r in range(min(2, len(invs))):
        compare(got[r:r + 1], q[r:r + 1], pg, r, int(pg.lens[r]) - 1, d, unit)
    got, cu = run_prefill(pg, qp, invs, bits, scale)
    for r in range(min(2, len(invs))):
        compare(got[cu[r]:cu[r + 1]], qp[cu[r]:cu[r + 1]], pg, r, invs[r][0], d, unit)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("name", list(INVOCATIONS))
def test_values_near_the_largest(name, d, bits):
    """|V| up to 2^127 (of one sign, and of both), whose weighted sums over hundreds of keys lie past
    float32 where the weights are not kept small; logits that rise by some tens after the first keys."""
    invs = INVOCATIONS[name]
    print(f"[case] large values, {name}, head_dim {d}, {bits} bits", flush=True)
    pg = QuantPaged(51, [p + s for p, s in invs], HKV, d, bits)
    pg.v = scaled(pg.v, 124)
    pg.v[:, 0] &= 0x7FFF
    for r in range(2):
        for j in range(33, pg.lens[r]):
            pg.k[pg.tables[r, j // 16], :, j % 16, 0] = 0x4000        # 2, and before 0
        for j in range(min(33, pg.lens[r])):
            pg.k[pg.tables[r, j // 16], :, j % 16, 0] = 0
    pg.requantise(bits)
    rng = pg.rng
    q, qp = bf16_bits(rng, len(invs), HQ, d), bf16_bits(rng, sum(s for _, s in invs), HQ, d)
    for x in (q, qp):
        x[:, :, 0] = 0x42A0                # 80: 160 scale in the logits, 14 or 20
    both(pg, q, qp, invs, bits, d, unit=2.0 ** 124)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("power", [-20, -40])
def test_small_values(d, bits, power):
    """V of 2^-20 and 2^-40: errors relative to that."""
    invs = INVOCATIONS["parts"]
    print(f"[case] values of 2^{power}, head_dim {d}, {bits} bits", flush=True)
    pg = QuantPaged(52, [p + s for p, s in invs], HKV, d, bits)
    pg.v = scaled(pg.v, power)
    pg.requantise(bits)
    rng = pg.rng
    q, qp = bf16_bits(rng, len(invs), HQ, d), bf16_bits(rng, sum(s for _, s in invs), HQ, d)
    both(pg, q, qp, invs, bits, d, unit=2.0 ** power)
