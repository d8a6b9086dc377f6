"""NaN in a pool held in 4 or 8 bits and in queries: which outputs it reaches, and that every other
one is right."""

import numpy as np
import pytest

from bounded_cache_util import bf16_bits
from quant_util import QuantPaged
from test_gpu_quant_attention import check_rows, run_decode, run_prefill

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

HQ, HKV = 8, 2
GROUP = HQ // HKV


def put(pool, pg, r, j, g, feature):
    pool[pg.tables[r, j // 16], g, j % 16, feature] = 0x7FC0


def head_rows(g):
    return slice(g * GROUP, (g + 1) * GROUP)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
def test_decode(d, bits):
    """A NaN key inside a sequence that several work-groups share makes the rows of its KV head NaN; a NaN
    group of V those rows' 32 features; what other sequences and KV heads give is right."""
    scale = float(np.float32(d ** -0.5))
    print(f"[case] NaN keys and values, decode, head_dim {d}, {bits} bits", flush=True)
    pg = QuantPaged(61, [9000, 1, 700, 40, 9001, 33], HKV, d, bits)
    put(pg.k, pg, 0, 4321, 1, 7)
    put(pg.k, pg, 1, 0, 0, 40)
    put(pg.v, pg, 2, 131, 0, 35)
    put(pg.v, pg, 3, 39, 1, 3)
    pg.requantise(bits)
    q = bf16_bits(pg.rng, 6, HQ, d)
    got = run_decode(pg, q, bits, scale)
    want = np.zeros((6, HQ, d), dtype=bool)
    want[0, head_rows(1)] = want[1, head_rows(0)] = True
    want[2, head_rows(0), 32:64] = want[3, head_rows(1), 0:32] = True
    assert (np.isnan(got) == want).all()
    for r in (0, 1, 2, 3, 4, 5):
        heads = [h for h in range(HQ) if not want[r, h].any()]
        check_rows(got[r:r + 1], q[r:r + 1], pg, r, int(pg.lens[r]) - 1, HQ, HKV, scale, heads)


# in parts of the keys, and more tiles than the device holds work-groups at once
BATCHES = {"parts": [(2000, 90), (0, 70), (500, 3)], "whole": [(300, 90), (0, 70), (500, 3)] + [(10, 700)] * 14}


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("name", list(BATCHES))
def test_prefill(name, d, bits):
    """A NaN key of the suffix reaches the rows from its own on, a prefix one every row; a NaN group of
    V of the prefix its 32 features of every row; a NaN group of V of the suffix those of the rows that see it,
    and of rows before at most those; a query with a NaN or an infinity its own row."""
    invs = BATCHES[name]
    scale = float(np.float32(d ** -0.5))
    print(f"[case] NaN, prefill, {name}, head_dim {d}, {bits} bits", flush=True)
    pg = QuantPaged(62, [p + s for p, s in invs], HKV, d, bits)
    p0, p2 = invs[0][0], invs[2][0]
    put(pg.k, pg, 0, p0 + 37, 0, 5)           # suffix key
    put(pg.v, pg, 0, p0 + 60, 1, 40)          # suffix value
    put(pg.v, pg, 2, p2 - 99, 0, 3)           # prefix value
    put(pg.k, pg, 2, 200, 1, 33)              # prefix key
    pg.requantise(bits)
    q = bf16_bits(pg.rng, sum(s for _, s in invs), HQ, d)
    q[90 + 11, 3, 50], q[90 + 69, 6, 0], q[90 + 30, 0, 9] = 0x7FC0, 0xFF80, 0x7F80
    got, cu = run_prefill(pg, q, invs, bits, scale)
    nan = np.isnan(got)
    want = np.zeros_like(nan)
    want[37:90, head_rows(0)] = True
    want[60:90, head_rows(1), 32:64] = True
    want[cu[2]:cu[3], head_rows(0), 0:32] = True
    want[cu[2]:cu[3], head_rows(1)] = True
    want[90 + 11, 3] = want[90 + 69, 6] = want[90 + 30, 0] = True
    may = want.copy()
    may[:60, head_rows(1), 32:64] = True
    assert (nan >= want).all(), "NaN is missing"
    assert (nan <= may).all(), "NaN where none may be"
    got = np.where(nan & ~want, 0.0, got)
    for r, (p, s) in enumerate(invs[:4]):
        for i in (range(s) if s <= 90 else (0, 1, 350, 699)):
            row = cu[r] + i
            heads = [h for h in range(HQ) if not may[row, h].any()]
            if heads:
                check_rows(got[row:row + 1], q[row:row + 1], pg, r, p + i, HQ, HKV, scale, heads)
