"""Random paged sequences for the tests of the operators that bound a cache."""

import numpy as np

BLOCK = 16
NAN_BITS = np.uint16(0x7FC0)


def bf16_bits(rng, *shape):
    """N(0, 1) as bf16 bit patterns."""
    x = rng.standard_normal(shape, dtype=np.float32).view(np.uint32)
    return ((x + 0x7FFF + ((x >> 16) & 1)) >> 16).astype(np.uint16)


class Paged:
    """Sequences of the given lengths in a pool of scattered slots, the last of which holds NaN:
    every table entry that no test reads names it.  The tables have room for `room` keys."""

    def __init__(self, seed, lens, hkv, d, spare=0, shared=0, room=0):
        rng = self.rng = np.random.default_rng(seed)
        blocks = [-(-n // BLOCK) for n in lens]
        used = shared + sum(max(0, b - shared) for b in blocks)
        self.num_blocks = used + spare + 3
        self.k = bf16_bits(rng, self.num_blocks, hkv, BLOCK, d)
        self.v = bf16_bits(rng, self.num_blocks, hkv, BLOCK, d)
        self.nan_slot = self.num_blocks - 1
        self.k[self.nan_slot] = self.v[self.nan_slot] = NAN_BITS
        order = rng.permutation(self.num_blocks - 1)
        self.free = list(order[used:])
        anchor, at = list(order[:shared]), shared
        self.tables = np.full((len(lens), max(max(blocks) + 1, -(-room // BLOCK))), self.nan_slot, dtype=np.int32)
        for r, b in enumerate(blocks):
            own = max(0, b - shared)
            self.tables[r, :b] = (anchor[:b] + list(order[at:at + own]))
            at += own
        self.lens = np.array(lens, dtype=np.int32)
        # past a sequence's end its last block holds what a recycled slot may hold
        for r, n in enumerate(lens):
            if n % BLOCK and blocks[r] > shared:
                self.k[self.tables[r, n // BLOCK], :, n % BLOCK:] = NAN_BITS
                self.v[self.tables[r, n // BLOCK], :, n % BLOCK:] = NAN_BITS

    def hide(self, r, sinks, low):
        """What sequence r does not see of its keys in [sinks, low) becomes NaN, and a block of such
        keys alone loses its table entry."""
        for b in range(self.tables.shape[1]):
            keys = np.arange(b * BLOCK, (b + 1) * BLOCK)
            gone = (keys >= sinks) & (keys < low)
            if gone.all():
                self.tables[r, b] = self.nan_slot
            elif gone.any():
                self.k[self.tables[r, b], :, gone] = NAN_BITS
                self.v[self.tables[r, b], :, gone] = NAN_BITS


def to_gpu(a):
    import torch
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint16:
        return torch.from_numpy(a.view(np.int16)).view(torch.bfloat16).cuda()
    return torch.from_numpy(a).cuda()


def to_bits(t):
    import torch
    return t.view(torch.int16).cpu().numpy().view(np.uint16)


def attention_bound(out, mag):
    """Largest error of a bf16 output, element by element.  The probabilities are rounded to bf16
    (half a step, 2^-8 of each) before their product with V and their sum, so an output is off
    by at most twice 2^-8 of sum w |v|, and is rounded once more; fp32 sums and logits (a dot
    product of 128 terms of about 100 in all: 1e-4 in the exponent at the worst) come on top."""
    return 2.0 ** -8 * (2 * mag + np.abs(out)) * 1.01 + 2e-4 * mag + 1e-6


def weight_bound(total):
    """Largest error of a sum of fp32 weights: an exponent's 1e-4 (as above) in the weight and in
    its normaliser."""
    return 2.1e-4 * np.abs(total) + 1e-7
