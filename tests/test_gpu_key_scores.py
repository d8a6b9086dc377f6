"""Attention weights added to scores, by decode and after a prefill, against the float64 oracle."""

import numpy as np
import pytest

from bounded_cache_util import Paged, attention_bound, bf16_bits, to_bits, to_gpu, weight_bound
from oracle import add_key_scores, bf16_bits_to_f64, window_attention

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def first_scores(pg, hkv):
    """Scores of the size that weights have; NaN where no key of the batch lies."""
    s = (pg.rng.random((pg.num_blocks, hkv, 16)) * 1e-2).astype(np.float32)
    s[pg.nan_slot] = np.nan
    return s


def run_decode(pg, q, scores, score_from, scale, decay, max_len=None, max_scored=None, workspace="auto",
               stream=None):
    from paper_2608_14624_amd import ops
    qd, sd = to_gpu(q), to_gpu(scores)
    out = torch.full_like(qd, float("nan"))
    scored = int(max(0, (pg.lens - score_from).max()))
    ops.cs_decode_attn_scores(qd, to_gpu(pg.k), to_gpu(pg.v), to_gpu(pg.tables), to_gpu(pg.lens),
                              to_gpu(score_from), sd, out, max_seq_len=max_len or int(pg.lens.max()),
                              max_scored_len=scored if max_scored is None else max_scored, scale=scale,
                              decay=decay, workspace=workspace, stream=stream)
    torch.cuda.synchronize()
    return to_bits(out), sd.cpu().numpy()


def check_decode(seed, hq, hkv, d, lens, froms, decay=1.0, shared=0, rows=None, **kw):
    scale = float(np.float32(d ** -0.5))
    print(f"[case] decode scores {hq}/{hkv} heads of {d}, lens {list(lens)[:8]} ({len(lens)}), from "
          f"{list(froms)[:8]}, decay {decay} {kw}", flush=True)
    pg = Paged(seed, lens, hkv, d, shared=shared)
    q = bf16_bits(pg.rng, len(lens), hq, d)
    old = first_scores(pg, hkv)
    froms = np.array(froms, dtype=np.int32)
    bits, new = run_decode(pg, q, old, froms, scale, decay, **kw)
    got = bf16_bits_to_f64(bits)
    # what a recycled slot held where the new token lies does not matter
    want = old.astype(np.float64)
    touched = np.zeros(old.shape, dtype=bool)
    for r, n in enumerate(lens):
        if n == 0:
            assert (bits[r] == 0).all(), "a row without keys is zero"
            continue
        j = np.arange(froms[r], n)
        touched[pg.tables[r, j // 16], :, j % 16] = True
        if rows is not None and r not in rows:
            want[pg.tables[r, j // 16], :, j % 16] = new[pg.tables[r, j // 16], :, j % 16]
            continue
        ref, mag = window_attention(q[r:r + 1], pg.k, pg.v, pg.tables[r], n - 1, hq, hkv, scale)
        err = np.abs(got[r:r + 1] - ref)
        assert np.isfinite(err).all() and (err <= attention_bound(ref, mag)).all(), f"sequence {r}: {err.max()}"
        add_key_scores(want, q[r:r + 1], pg.k, pg.tables[r], n - 1, n - 1, int(froms[r]), hq, hkv, scale,
                       float(np.float32(decay)))
    assert (new.view(np.int32)[~touched] == old.view(np.int32)[~touched]).all(), "an unscored slot changed"
    err = np.abs(new - want)[touched]
    assert (err <= weight_bound(want[touched])).all(), f"scores off by {err.max()}"


LENS = [1000, 0, 1, 15, 16, 17, 31, 32, 33, 64, 0, 127, 129, 640, 999]


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64), (5, 1, 128), (16, 1, 64), (6, 3, 64)])
def test_decode_ragged_lengths(hq, hkv, d):
    check_decode(31, hq, hkv, d, LENS, [0] * len(LENS), decay=0.9)


@pytest.mark.parametrize("d", [64, 128])
def test_decode_scored_from_anywhere(d):
    froms = [0, 5, 1, 3, 31, 0, 17, 33, 40, 13, 2, 126, 128, 640, 997]
    check_decode(32, 8, 2, d, LENS, froms)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[1], [5, 0, 128], [100, 37, 64, 120]])
def test_decode_short(lens, d):
    """One work-group per sequence and KV head."""
    check_decode(33, 8, 2, d, lens, [min(3, n) for n in lens], decay=0.5)


def test_decode_more_sequences_than_a_plan_takes():
    lens = [(11 * i) % 190 for i in range(1100)]
    check_decode(34, 4, 1, 64, lens, [i % 7 for i in range(1100)], rows=[0, 1, 2, 300, 777, 1099])


def test_decode_one_long_sequence():
    check_decode(35, 8, 1, 128, [20011], [37])


def test_decode_full_batch_on_a_shared_anchor():
    """Sequences on one anchor, scored past it: pieces cut at the same places."""
    lens = [1200 + 13 * i for i in range(64)]
    check_decode(36, 32, 8, 128, lens, [960] * 64, shared=60, rows=[0, 1, 40, 63], decay=0.97)


@pytest.mark.parametrize("hq,hkv,d,batch", [(32, 8, 128, 41), (32, 8, 64, 33), (40, 8, 128, 32), (16, 16, 64, 20)])
def test_decode_a_work_group_per_pair(hq, hkv, d, batch):
    """At least as many sequences and KV heads as compute units."""
    lens = [(397 * i) % 1300 for i in range(batch)]
    check_decode(46, hq, hkv, d, lens, [(5 * i) % 200 for i in range(batch)], decay=0.7, rows=[0, 1, 2, batch // 2, batch - 1])


def test_decode_more_logits_than_a_compute_unit_holds():
    """16 query heads per KV head: past about 1900 scored keys their logits go to the workspace."""
    lens = [4000, 2500, 1800, 0] + [60] * 29
    check_decode(47, 128, 8, 128, lens, [33, 0, 5, 0] + [0] * 29, rows=[0, 1, 2, 32])


def test_decode_batch_in_its_own_order():
    """More sequences than are ordered by length, one work-group per sequence and KV head."""
    lens = [(61 * i) % 250 + 1 for i in range(300)]
    check_decode(48, 8, 1, 64, lens, [0] * 300, rows=[0, 7, 299])


def test_decode_nothing_scored():
    check_decode(37, 8, 2, 128, [300, 40], [300, 100])


def test_decode_loose_bounds_and_a_larger_workspace():
    ws = torch.empty(1 << 25, dtype=torch.uint8, device="cuda")
    check_decode(38, 8, 2, 128, [300, 40, 0], [7, 0, 0], max_len=312, max_scored=310, workspace=ws)


def test_decode_scores_past_their_bound_are_left():
    """max_scored_len is a bound of the caller's: keys past it keep their scores."""
    pg = Paged(39, [900], 2, 128)
    q = bf16_bits(pg.rng, 1, 8, 128)
    old = first_scores(pg, 2)
    print("[case] decode scores past their bound", flush=True)
    _, new = run_decode(pg, q, old, np.array([0], dtype=np.int32), 0.09, 1.0, max_scored=200)
    j = np.arange(300, 900)
    at = (pg.tables[0, j // 16], slice(None), j % 16)
    assert (new[at] == old[at]).all()


def check_prefill(seed, hq, hkv, d, invs, froms, rows, decay=1.0, max_q=None, max_kv=None, workspace="auto",
                  only=None, stream=None):
    from paper_2608_14624_amd import ops
    scale = float(np.float32(d ** -0.5))
    print(f"[case] prefill scores {hq}/{hkv} heads of {d}, {invs[:4]}.. ({len(invs)}), from {froms[:4]}, rows {rows}, "
          f"decay {decay}", flush=True)
    pg = Paged(seed, [p + s for p, s in invs], hkv, d)
    q = bf16_bits(pg.rng, sum(s for _, s in invs), hq, d)
    cu = np.concatenate([[0], np.cumsum([s for _, s in invs])]).astype(np.int32)
    old = first_scores(pg, hkv)
    sd = to_gpu(old)
    ops.cs_prefill_key_scores(to_gpu(q), to_gpu(pg.k), to_gpu(pg.tables),
                              to_gpu(np.array([p for p, _ in invs], dtype=np.int32)), to_gpu(cu),
                              to_gpu(np.array(froms, dtype=np.int32)), sd,
                              max_q_len=max_q or max(s for _, s in invs),
                              max_kv_len=max_kv or max(p + s for p, s in invs), rows=rows, scale=scale,
                              decay=decay, workspace=workspace, stream=stream)
    torch.cuda.synchronize()
    new = sd.cpu().numpy()
    want = old.astype(np.float64)
    touched = np.zeros(old.shape, dtype=bool)
    for r, (p, s) in enumerate(invs):
        if s == 0:
            continue
        n = min(s, rows)
        j = np.arange(froms[r], p + s)
        touched[pg.tables[r, j // 16], :, j % 16] = True
        if only is not None and r not in only:
            want[pg.tables[r, j // 16], :, j % 16] = new[pg.tables[r, j // 16], :, j % 16]
            continue
        add_key_scores(want, q[cu[r + 1] - n:cu[r + 1]], pg.k, pg.tables[r], p + s - n, p, froms[r], hq, hkv,
                       scale, float(np.float32(decay)))
    assert (new.view(np.int32)[~touched] == old.view(np.int32)[~touched]).all(), "an unscored slot changed"
    err = np.abs(new - want)[touched]
    assert (err <= weight_bound(want[touched])).all(), f"scores off by {err.max()}"


INVS = [(300, 70), (0, 130), (517, 1), (64, 0), (0, 1), (31, 33)]
FROMS = [288, 0, 3, 0, 0, 40]


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64), (5, 1, 128), (16, 1, 64), (6, 3, 128), (20, 1, 64)])
@pytest.mark.parametrize("rows", [1, 2, 32, 33, 1000])
def test_prefill_ragged(hq, hkv, d, rows):
    check_prefill(41, hq, hkv, d, INVS, FROMS, rows, decay=0.8)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [16, 400])
def test_prefill_key_parts(d, rows):
    """Few rows on a long sequence: their statistics come from several key parts."""
    check_prefill(42, 8, 2, d, [(4000, 40), (2500, 500)], [0, 2496], rows)


def test_prefill_many_rows():
    check_prefill(43, 32, 8, 128, [(300, 900), (0, 700), (80, 1000)], [288, 0, 80], 5000, only=[1])


def test_prefill_loose_bounds_and_a_larger_workspace():
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    check_prefill(44, 8, 2, 128, [(100, 30), (0, 20)], [0, 0], 25, max_q=64, max_kv=144, workspace=ws)


def test_prefill_of_one_token_is_the_decode():
    """The scores of a one-token suffix are those that decode adds."""
    from paper_2608_14624_amd import ops
    hq, hkv, d, n = 8, 2, 128, 777
    pg = Paged(45, [n], hkv, d)
    q = bf16_bits(pg.rng, 1, hq, d)
    old = first_scores(pg, hkv)
    print("[case] one-token prefill scores against decode", flush=True)
    zero = np.array([0], dtype=np.int32)
    _, by_decode = run_decode(pg, q, old, zero, 0.09, 0.5)
    sd = to_gpu(old)
    ops.cs_prefill_key_scores(to_gpu(q), to_gpu(pg.k), to_gpu(pg.tables), to_gpu(zero + n - 1),
                              to_gpu(np.array([0, 1], dtype=np.int32)), to_gpu(zero), sd, max_q_len=1,
                              max_kv_len=n, rows=1, scale=0.09, decay=0.5)
    torch.cuda.synchronize()
    np.testing.assert_allclose(sd.cpu().numpy(), by_decode, rtol=1e-4, atol=1e-7, equal_nan=True)


@pytest.mark.parametrize("lens", [[3000, 45], [1501 + i for i in range(130)]])
@pytest.mark.parametrize("beyond", [0, 1, 3, 2 ** 31 - 1])
def test_decode_scored_from_its_end_or_beyond(lens, beyond):
    """Nothing of the first sequence is scored, however far past its end score_from lies, in ranges
    and by pairs; the others are as ever."""
    froms = [min(lens[0] + beyond, 2 ** 31 - 1)] + [7] * (len(lens) - 1)
    check_decode(49, 8, 2, 128, lens, froms, max_scored=max(lens), rows=[0, 1])


@pytest.mark.parametrize("rows", [5, 400])
@pytest.mark.parametrize("beyond", [0, 1, 2 ** 31 - 1])
def test_prefill_scored_from_its_end_or_beyond(rows, beyond):
    check_prefill(50, 32, 8, 128, [(1700, 405), (0, 390)], [min(2105 + beyond, 2 ** 31 - 1), 3], rows)


@pytest.mark.parametrize("lens", [[9000] + [40 + i for i in range(31)], [6144 - i for i in range(32)]])
def test_decode_of_a_batch_that_one_sequence_may_dominate(lens):
    """Both sides of the bound on the longest sequence up to which a work-group takes a whole one."""
    check_decode(52, 16, 8, 128, lens, [3] * 32, rows=[0, 31], decay=0.8)
