"""Random sequences in a pool held in 4 or 8 bits, for its tests."""

import numpy as np

from bounded_cache_util import Paged
from oracle import bf16_bits_to_f64, pack_tiles, to_bf16_bits, unpack_tiles


def spread_rows(rng, *shape):
    """bf16 bits of rows whose groups of 32 features lie in different powers of two, with zeros, a
    few large features and signed zeros among them."""
    x = rng.standard_normal(shape) * np.exp2(rng.integers(-6, 7, size=(*shape[:-1], shape[-1] // 32)).repeat(32, -1))
    x[rng.random(shape) < 0.02] *= 8
    x[rng.random(shape) < 0.02] = 0.0
    x[rng.random(shape) < 0.02] *= -0.0
    return (x.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)


class QuantPaged(Paged):
    """Paged sequences whose pools are quantised: ``tiles`` as the calls take them, k and v the bf16
    numbers that they hold.  What lies behind a sequence's end, and a last slot, are NaN."""

    def __init__(self, seed, lens, hkv, d, bits, **kw):
        super().__init__(seed, lens, hkv, d, **kw)
        self.requantise(bits)

    def requantise(self, bits):
        d = self.k.shape[-1]
        self.tiles = pack_tiles(self.k, self.v, bits)
        self.k, self.v = (to_bf16_bits(x) for x in unpack_tiles(self.tiles, d, bits))


def quant_attention_bound(out, mag):
    """Largest error of a bf16 output, element by element: every probability is rounded to bf16 (half
    a step, 2^-8 of it) for its product with V, and the output once more; the sum of the
    probabilities is not.  fp32 sums and logits (a dot product of 128 terms of about 100 in all:
    1e-4 in the exponent at the worst) come on top."""
    return 2.0 ** -8 * (mag + np.abs(out)) * 1.01 + 2e-4 * mag + 1e-6


def f64(bits):
    return bf16_bits_to_f64(bits)
