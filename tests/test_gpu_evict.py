"""Eviction within sequences against the oracle: the kept keys, K, V and scores are exact."""

import numpy as np
import pytest

from bounded_cache_util import NAN_BITS, Paged, to_bits, to_gpu
from oracle import evict

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

SCORES = {
    "spread": lambda rng, shape: np.exp(3 * rng.standard_normal(shape)),
    "all equal": lambda rng, shape: np.full(shape, 0.25),
    "many ties": lambda rng, shape: rng.integers(0, 5, shape) * 0.5,
    "near": lambda rng, shape: 1 + rng.integers(0, 4000, shape) * 2.0 ** -23,
    "zeros of both signs": lambda rng, shape: rng.choice([0.0, -0.0, 1e-45, -1.0], shape),
    "special": lambda rng, shape: rng.choice([np.inf, -np.inf, np.nan, 1.0, -3.0, 0.0], shape),
}


def check(seed, hkv, d, lens, froms, budget, trigger, recent, kind="spread", moving=False, max_len=None,
          in_place_lens=False, stream=None):
    from paper_2608_14624_amd import ops
    print(f"[case] evict {hkv} heads of {d}, lens {list(lens)[:6]} ({len(lens)}), from {list(froms)[:6]}, budget {budget}, "
          f"trigger {trigger}, recent {recent}, scores {kind}, {'other' if moving else 'own'} blocks", flush=True)
    per_seq = -(-(budget + 15) // 16) + 1
    pg = Paged(seed, lens, hkv, d, spare=per_seq * len(lens) if moving else 0)
    width = max(pg.tables.shape[1], (max(froms) + budget) // 16 + 2)
    tables = np.full((len(lens), width), pg.nan_slot, dtype=np.int32)
    tables[:, :pg.tables.shape[1]] = pg.tables
    dst = None
    if moving:
        dst = tables.copy()
        for r, f in enumerate(froms):
            n = -(-(f + budget) // 16) - f // 16
            dst[r, f // 16:] = pg.nan_slot
            dst[r, f // 16:f // 16 + n] = [pg.free.pop() for _ in range(n)]
    scores = SCORES[kind](pg.rng, (pg.num_blocks, hkv, 16)).astype(np.float32)
    lens32, from32 = np.array(lens, dtype=np.int32), np.array(froms, dtype=np.int32)
    kd, vd, sd, ld = to_gpu(pg.k), to_gpu(pg.v), to_gpu(scores), to_gpu(lens32)
    kept = torch.full((len(lens), hkv, budget), -7, dtype=torch.int32, device="cuda")
    new_lens = ld if in_place_lens else torch.full_like(ld, -7)
    ops.cs_kv_evict(sd, kd, vd, to_gpu(tables), None if dst is None else to_gpu(dst), ld, to_gpu(from32), kept,
                    new_lens, max_seq_len=max_len or max(lens), budget=budget, trigger=trigger, recent=recent,
                    stream=stream)
    torch.cuda.synchronize()
    k, v, s = pg.k.copy(), pg.v.copy(), scores.copy()
    want_lens, want_kept = [], np.full((len(lens), hkv, budget), -7, dtype=np.int32)
    for r, n in enumerate(lens):
        got, new = evict(s, k, v, tables[r], None if dst is None else dst[r], n, froms[r], budget, trigger, recent)
        want_lens.append(new)
        if got is None:
            want_kept[r, :, 0] = -1
        else:
            want_kept[r] = got
    assert new_lens.cpu().numpy().tolist() == want_lens
    assert (kept.cpu().numpy() == want_kept).all()
    assert (to_bits(kd) == k).all() and (to_bits(vd) == v).all()
    assert (sd.cpu().numpy().view(np.int32) == s.view(np.int32)).all()
    assert (k[pg.nan_slot] == NAN_BITS).all()


@pytest.mark.parametrize("moving", [False, True])
@pytest.mark.parametrize("kind", sorted(SCORES))
def test_choices(kind, moving):
    check(51, 2, 128, [700, 333, 40], [0, 5, 16], 100, 100, 20, kind, moving)


@pytest.mark.parametrize("moving", [False, True])
@pytest.mark.parametrize("budget,trigger,recent", [(1, 1, 0), (1, 1, 1), (16, 16, 16), (17, 40, 0), (300, 300, 299),
                                                    (511, 513, 7), (512, 512, 0), (999, 999, 500)])
def test_budgets(budget, trigger, recent, moving):
    lens = [0, 1, 2, 17, 41, 515, 1000, 1001, 1300]
    check(52, 3, 64, lens, [0, 0, 1, 0, 0, 1, 1, 0, 33], budget, trigger, recent, "many ties", moving)


@pytest.mark.parametrize("moving", [False, True])
def test_one_key_goes(moving):
    check(53, 8, 128, [258, 259], [2, 2], 256, 256, 3, "spread", moving)


@pytest.mark.parametrize("moving", [False, True])
def test_long(moving):
    check(54, 2, 128, [30011, 9000], [100, 2048], 4097, 5000, 64, "spread", moving, max_len=30016)


def test_nothing_to_evict_and_lengths_in_place():
    check(55, 2, 64, [50, 300, 0], [10, 0, 0], 60, 90, 4, in_place_lens=True)


def test_more_kept_than_fits_a_chunk_in_place():
    """The copy within a sequence's own blocks goes by chunks of kept keys."""
    check(56, 1, 64, [9000], [3], 6000, 6000, 1, "near")
