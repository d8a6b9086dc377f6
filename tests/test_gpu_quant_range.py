"""Attention over a pool held in 4 or 8 bits at the ends of the numbers' range: values near the
format's largest and far below 1, and logits past 2^31, where float32 holds no fractions."""

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
    """bf16 bits of numbers times 2^power, exactly, but for those that would be subnormal: zeros; NaN as it is."""
    exponent = (bits >> 7 & 0xFF).astype(np.int32)
    x = np.where(exponent + power > 0, bits + np.uint16(power << 7 & 0xFFFF), bits & 0x8000)
    return np.where((exponent == 0) | (exponent == 255), bits, x).astype(np.uint16)


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


def huge_logits(pg, d, rows, exponents, sign):
    """Queries of one feature, so that a key's logit is that feature's product: K of +-2^e with e from
    `exponents` by position.  Logits are then equal or at least twice as large, in any arithmetic."""
    q = np.zeros((rows, HQ, d), dtype=np.uint16)
    q[:, :, 0] = 0x3FB0 + (10 << 7)                      # 1.375 * 2^10
    q[:, 1::2, 0] |= 0x8000
    for r, n in enumerate(pg.lens):
        for j in range(n):
            e = exponents(j, n)
            x = np.uint16((127 + e) << 7) | (0x8000 if sign(j) else 0)
            pg.k[pg.tables[r, j // 16], :, j % 16, 0] = x
    return q


HUGE = {
    "equal": (lambda j, n: 24, lambda j: False),
    "equal, 2^31": (lambda j, n: 21, lambda j: False),
    "equal and far": (lambda j, n: 100, lambda j: False),
    "both signs": (lambda j, n: 30, lambda j: j % 5 == 2),
    "rising": (lambda j, n: -20 + 80 * j // n, lambda j: False),
    "falling": (lambda j, n: 60 - 80 * j // n, lambda j: False),
    "mixed": (lambda j, n: 20 + j * 37 % 23, lambda j: j % 3 == 0),
}


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("name", list(HUGE))
def test_logits_past_float32s_whole_numbers(name, d, bits):
    """The result is the mean of V over the largest logit's keys (a single key's V where there is one)."""
    exponents, sign = HUGE[name]
    invs = [(0, 1), (0, 5), (300, 2), (900, 70)]
    print(f"[case] huge logits, {name}, head_dim {d}, {bits} bits", flush=True)
    pg = QuantPaged(53, [p + s for p, s in invs], HKV, d, bits)
    q = huge_logits(pg, d, len(invs), exponents, sign)
    qp = huge_logits(pg, d, sum(s for _, s in invs), exponents, sign)
    pg.requantise(bits)
    scale = float(np.float32(d ** -0.5))
    got = run_decode(pg, q, bits, scale)
    for r, n in enumerate(pg.lens):
        compare(got[r:r + 1], q[r:r + 1], pg, r, int(n) - 1, d)
    got, cu = run_prefill(pg, qp, invs, bits, scale)
    for r, (p, s) in enumerate(invs):
        compare(got[cu[r]:cu[r + 1]], qp[cu[r]:cu[r + 1]], pg, r, p, d)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
def test_a_large_feature_that_all_keys_share(d, bits):
    """A channel of 32 in every key and of +-128 in every query, as biased projections have them: its
    product, 4096, is the same for all keys, and the 31 features of its group decide the weights.  A logit is a sum of
    up to 128 products that fp32 holds to 2^-24 of some 2^13 each, 2^-4 scale at the worst."""
    scale = float(np.float32(d ** -0.5))
    print(f"[case] a large shared feature, head_dim {d}, {bits} bits", flush=True)
    invs = [(600, 40), (0, 33), (2000, 3)]
    pg = QuantPaged(55, [p + s for p, s in invs], HKV, d, bits)
    rng = pg.rng
    pg.k[..., 1:32] = scaled(pg.k[..., 1:32], 3)
    pg.k[..., 0] = np.where(pg.k[..., 0] == 0x7FC0, pg.k[..., 0], 0x4200)
    pg.requantise(bits)
    q, qp = bf16_bits(rng, len(invs), HQ, d), bf16_bits(rng, sum(s for _, s in invs), HQ, d)
    for x in (q, qp):
        x[..., 0] = 0x4300 | (x[..., 0] & 0x8000)

    def check(got, q, r, first):
        slack = np.expm1(2 * scale * 2.0 ** -4)
        out, mag = window_attention(q, pg.k, pg.v, pg.tables[r], first, HQ, HKV, scale)
        worst = float((np.abs(got - out) / (quant_attention_bound(out, mag) + slack * (mag + np.abs(out)))).max())
        assert worst <= 1, f"{worst} of the bound"

    got = run_decode(pg, q, bits, scale)
    for r, n in enumerate(pg.lens):
        check(got[r:r + 1], q[r:r + 1], r, int(n) - 1)
    got, cu = run_prefill(pg, qp, invs, bits, scale)
    for r, (p, _) in enumerate(invs):
        check(got[cu[r]:cu[r + 1]], qp[cu[r]:cu[r + 1]], r, p)
