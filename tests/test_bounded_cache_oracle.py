"""The float64 oracles of windowed attention, key scores and eviction: pinned to the attention
oracle, to scalar loops and to hand-worked cases, with planted mistakes that the pins find."""

import math

import numpy as np
import pytest

import oracle
import oracle.bounded_cache as bc
from bounded_cache_util import Paged, bf16_bits


def scalar_window_row(q, k, v, p, scale, window, sinks):
    """One row by scalar loops."""
    seen = [j for j in range(p + 1) if j > p - window or j < sinks]
    logits = [scale * sum(float(a) * float(b) for a, b in zip(q, k[j])) for j in seen]
    top = max(logits)
    w = [math.exp(x - top) for x in logits]
    return [sum(wi * float(v[j][d]) for wi, j in zip(w, seen)) / sum(w) for d in range(len(q))]


def check_window(window, sinks, prefix=19, rows=23):
    hq, hkv, d = 4, 2, 8
    pg = Paged(5, [prefix + rows], hkv, d)
    q = bf16_bits(pg.rng, rows, hq, d)
    scale = np.float32(0.3)
    out, _ = bc.window_attention(q, pg.k, pg.v, pg.tables[0], prefix, hq, hkv, scale, window, sinks)
    qf, kf, vf = (oracle.bf16_bits_to_f64(x) for x in (q, pg.k, pg.v))
    at = [(pg.tables[0, j // 16], j % 16) for j in range(prefix + rows)]
    for i in range(rows):
        for h in range(hq):
            k = [kf[b, h // 2, o] for b, o in at]
            v = [vf[b, h // 2, o] for b, o in at]
            want = scalar_window_row(qf[i, h], k, v, prefix + i, float(scale), window, sinks)
            np.testing.assert_allclose(out[i, h], want, rtol=0, atol=1e-12)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (5, 0), (7, 4), (16, 16), (30, 40), (100, 0)])
def test_window_is_the_scalar_definition(window, sinks):
    check_window(window, sinks)


def test_a_window_over_everything_is_the_attention_oracle():
    pg = Paged(6, [45], 2, 8)
    q = bf16_bits(pg.rng, 20, 4, 8)
    ref = oracle.prefill_paged_attn(q, pg.k, pg.v, pg.tables, np.array([25]), np.array([0, 20]), 4, 2, 0.25)
    out, _ = bc.window_attention(q, pg.k, pg.v, pg.tables[0], 25, 4, 2, 0.25, 45, 0)
    np.testing.assert_allclose(out, ref, rtol=0, atol=1e-12)


def test_weights_of_every_row_sum_to_one_per_head():
    pg = Paged(7, [40], 2, 8)
    q = bf16_bits(pg.rng, 9, 6, 8)
    scores = np.zeros((pg.num_blocks, 2, 16))
    bc.add_key_scores(scores, q, pg.k, pg.tables[0], 31, 31, 0, 6, 2, 0.4, 0.5)
    np.testing.assert_allclose(scores.sum((0, 2)), [9 * 3] * 2, rtol=1e-12)


def test_scores_decay_start_anew_and_leave_the_rest():
    pg = Paged(8, [33], 1, 8)
    q = bf16_bits(pg.rng, 3, 2, 8)
    old = pg.rng.random((pg.num_blocks, 1, 16))
    added = np.zeros_like(old)
    bc.add_key_scores(added, q, pg.k, pg.tables[0], 30, 0, 0, 2, 1, 0.4, 1.0)
    new = old.copy()
    bc.add_key_scores(new, q, pg.k, pg.tables[0], 30, 30, 5, 2, 1, 0.4, 0.75)
    for j in range(48):
        at = (pg.tables[0, j // 16], 0, j % 16)
        want = old[at] if j < 5 or j >= 33 else added[at] + (0.75 * old[at] if j < 30 else 0)
        assert new[at] == pytest.approx(want, abs=1e-12)


def test_eviction_by_hand():
    pg = Paged(9, [20], 1, 8, spare=2)
    pg.tables[0, 2] = pg.free[0]
    scores = np.zeros((pg.num_blocks, 1, 16))
    own = {4: 1.0, 5: 3.0, 6: 2.0, 7: 2.0, 8: 0.5, 9: 2.0, 18: 0.0, 19: 0.0}
    for j, x in own.items():
        scores[pg.tables[0, j // 16], 0, j % 16] = x
    k0 = pg.k.copy()
    kept, n = bc.evict(scores, pg.k, pg.v, pg.tables[0], None, 20, 4, 5, 15, 2)
    assert kept.tolist() == [[5, 6, 7, 18, 19]] and n == 9        # of 6, 7 and 9 the first two
    for i, j in enumerate(kept[0]):
        assert (pg.k[pg.tables[0, 0], 0, 4 + i] == k0[pg.tables[0, j // 16], 0, j % 16]).all()
    assert scores[pg.tables[0, 0], 0, 4:9].tolist() == [3.0, 2.0, 2.0, 0.0, 0.0]
    assert bc.evict(scores, pg.k, pg.v, pg.tables[0], None, 20, 4, 5, 16, 2) == (None, 20)


def test_eviction_into_other_blocks_takes_the_keys_before():
    pg = Paged(10, [60], 2, 8, spare=4)
    dst = pg.tables[0].copy()
    dst[1:3] = pg.free[:2]
    scores = pg.rng.random((pg.num_blocks, 2, 16))
    k0 = pg.k.copy()
    kept, n = bc.evict(scores, pg.k, pg.v, pg.tables[0], dst, 60, 19, 10, 20, 0)
    assert n == 29
    for g in range(2):
        for j in range(16, 29):
            src = j if j < 19 else kept[g][j - 19]
            assert (pg.k[dst[j // 16], g, j % 16] == k0[pg.tables[0, src // 16], g, src % 16]).all()
    rest = [b for b in range(pg.num_blocks) if b not in dst[1:3]]
    assert (pg.k[rest] == k0[rest]).all()


@pytest.mark.parametrize("wrong", ["window one short", "window one long", "sinks dropped", "wrong head"])
def test_planted_mistakes_are_found(wrong, monkeypatch):
    weights = bc.window_weights

    def bad(q, k_pool, table, first_pos, num_rows, g, group, scale, window=None, sinks=0):
        if wrong == "window one short":
            window = max(1, window - 1)
        elif wrong == "window one long":
            window += 1
        elif wrong == "sinks dropped":
            sinks = 0
        else:
            g = 0
        return weights(q, k_pool, table, first_pos, num_rows, g, group, scale, window, sinks)
    monkeypatch.setattr(bc, "window_weights", bad)
    with pytest.raises(AssertionError):
        check_window(7, 4)
