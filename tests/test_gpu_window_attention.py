"""Prefill and decode attention with a sliding window and sinks against the float64 oracle:
every kernel a call can get, windows from one key to more than all, lengths from zero on, with NaN
in every key, block and table entry that no row sees."""

import numpy as np
import pytest

from bounded_cache_util import Paged, attention_bound, bf16_bits, to_bits, to_gpu
from oracle import bf16_bits_to_f64, window_attention

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def prefill_batch(seed, hq, hkv, d, invs, window, sinks, room=0):
    """(prefix, suffix) per invocation; what none of an invocation's rows sees is poisoned."""
    pg = Paged(seed, [p + s for p, s in invs], hkv, d, room=room)
    for r, (p, s) in enumerate(invs):
        pg.hide(r, sinks, p - window + 1 if s else p)
    q = bf16_bits(pg.rng, sum(s for _, s in invs), hq, d)
    return pg, q


def run_prefill(pg, q, invs, window, sinks, scale, workspace="auto", max_q=None, max_kv=None, stream=None):
    from paper_2608_14624_amd import ops
    cu = np.concatenate([[0], np.cumsum([s for _, s in invs])]).astype(np.int32)
    qd = to_gpu(q)
    out = torch.full_like(qd, float("nan"))
    ops.cs_prefill_window_attn(
        qd, to_gpu(pg.k), to_gpu(pg.v), to_gpu(pg.tables),
        to_gpu(np.array([p for p, _ in invs], dtype=np.int32)), to_gpu(cu), out,
        max_q_len=max_q or max(s for _, s in invs), max_kv_len=max_kv or max(p + s for p, s in invs),
        window=window, sinks=sinks, scale=scale, workspace=workspace, stream=stream)
    torch.cuda.synchronize()
    return bf16_bits_to_f64(to_bits(out)), cu


def check_prefill(seed, hq, hkv, d, invs, window, sinks, heads=None, rows=None, **kw):
    scale = float(np.float32(d ** -0.5))
    print(f"[case] window prefill {hq}/{hkv} heads of {d}, {invs[:4]}.. ({len(invs)}), window {window}, "
          f"sinks {sinks} {kw}", flush=True)
    pg, q = prefill_batch(seed, hq, hkv, d, invs, window, sinks, kw.get("max_kv") or 0)
    got, cu = run_prefill(pg, q, invs, window, sinks, scale, **kw)
    heads = range(hq) if heads is None else heads
    for r, (p, s) in enumerate(invs):
        if s == 0 or (rows is not None and r not in rows):
            continue
        out, mag = window_attention(q[cu[r]:cu[r + 1]], pg.k, pg.v, pg.tables[r], p, hq, hkv, scale, window,
                                    sinks, heads)
        err = np.abs(got[cu[r]:cu[r + 1]][:, list(heads)] - out)
        assert np.isfinite(err).all(), f"invocation {r}: non-finite output"
        assert (err <= attention_bound(out, mag)).all(), f"invocation {r}: {err.max()}"


# less than a round of ping-pong tiles: split tiles (and key parts, where the window is long)
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64), (5, 1, 128), (16, 1, 64), (6, 3, 128)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 5), (17, 0), (64, 64), (100, 4), (333, 70), (5000, 3)])
def test_split_tiles(hq, hkv, d, window, sinks):
    check_prefill(11, hq, hkv, d, [(300, 70), (0, 130), (517, 1), (64, 0), (0, 1), (31, 33)], window, sinks)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks,workspace", [(1500, 4, "auto"), (1500, 4, None), (1999, 200, "auto"),
                                                     (1, 1900, "auto"), (1200, 0, "auto")])
def test_key_parts(d, window, sinks, workspace):
    """Few rows on long sequences: the keys in sight are cut into parts (without a workspace
    tensor of the right size the call is refused, so None stands for one that is larger)."""
    if workspace is None:
        workspace = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    check_prefill(12, 8, 2, d, [(2100, 20), (1990, 35)], window, sinks, workspace=workspace)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(1, 0), (100, 3), (130, 0), (600, 100)])
def test_ping_pong_equal_suffixes(d, window, sinks):
    """32 query heads of 8: tiles of 64 tokens, 8 KV heads: more than a round of tiles."""
    check_prefill(13, 32, 8, d, [(700, 1100), (0, 1100)], window, sinks, heads=[0, 13, 31])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(37, 9), (512, 0), (256, 300)])
def test_ping_pong_ragged(d, window, sinks):
    invs = [(500, 900), (0, 1300), (80, 3), (0, 0), (1200, 700), (33, 65), (0, 640)]
    check_prefill(14, 32, 8, d, invs, window, sinks, heads=[5, 30])


def test_many_rounds_ragged_d64():
    """Past the rounds from which head_dim 64 goes without half tiles."""
    invs = [(300 + 7 * i, 200 + 61 * (i % 9)) for i in range(40)]
    check_prefill(15, 32, 8, 64, invs, 150, 4, heads=[3, 28], rows=[0, 8, 39])


def test_loose_bounds():
    check_prefill(16, 8, 2, 128, [(300, 70), (0, 40)], 90, 8, max_q=500, max_kv=590)


def test_a_window_over_everything_is_the_call_without():
    from paper_2608_14624_amd import ops
    invs = [(700, 90), (0, 60)]
    pg = Paged(17, [p + s for p, s in invs], 8, 128)
    q = bf16_bits(pg.rng, 150, 32, 128)
    print("[case] window over everything", flush=True)
    got, cu = run_prefill(pg, q, invs, 790, 0, 0.1)
    qd = to_gpu(q)
    ref = torch.full_like(qd, float("nan"))
    ops.cs_prefill_paged_attn(qd, to_gpu(pg.k), to_gpu(pg.v), to_gpu(pg.tables),
                              to_gpu(np.array([700, 0], dtype=np.int32)), to_gpu(cu), ref, max_q_len=90,
                              max_kv_len=790, scale=0.1, workspace="auto")
    torch.cuda.synchronize()
    assert (got == bf16_bits_to_f64(to_bits(ref))).all()


def check_decode(seed, hq, hkv, d, lens, window, sinks, max_len=None, shared=0, rows=None, stream=None):
    from paper_2608_14624_amd import ops
    scale = float(np.float32(d ** -0.5))
    print(f"[case] window decode {hq}/{hkv} heads of {d}, lens {list(lens)[:8]} ({len(lens)}), window {window}, "
          f"sinks {sinks}", flush=True)
    pg = Paged(seed, lens, hkv, d, shared=shared, room=max_len or 0)
    if shared == 0:
        for r, n in enumerate(lens):
            pg.hide(r, sinks, n - window)
    q = bf16_bits(pg.rng, len(lens), hq, d)
    qd = to_gpu(q)
    out = torch.full_like(qd, float("nan"))
    ops.cs_decode_window_attn(qd, to_gpu(pg.k), to_gpu(pg.v), to_gpu(pg.tables), to_gpu(pg.lens), out,
                              max_seq_len=max_len or max(lens), window=window, sinks=sinks, scale=scale,
                              stream=stream)
    torch.cuda.synchronize()
    got = bf16_bits_to_f64(to_bits(out))
    for r, n in enumerate(lens):
        if rows is not None and r not in rows:
            continue
        if n == 0:
            assert (to_bits(out[r]) == 0).all(), "a row without keys is zero"
            continue
        ref, mag = window_attention(q[r:r + 1], pg.k, pg.v, pg.tables[r], n - 1, hq, hkv, scale, window, sinks)
        err = np.abs(got[r:r + 1] - ref)
        assert np.isfinite(err).all() and (err <= attention_bound(ref, mag)).all(), f"sequence {r}: {err.max()}"


LENS = [1000, 0, 1, 15, 16, 17, 31, 32, 33, 64, 0, 127, 129, 640, 999, 0]


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64), (5, 1, 128), (16, 1, 64)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (33, 7), (100, 40), (130, 0), (500, 33),
                                           (999, 0), (1000, 0), (4000, 9)])
def test_decode(hq, hkv, d, window, sinks):
    check_decode(21, hq, hkv, d, LENS, window, sinks)


@pytest.mark.parametrize("window,sinks", [(1000, 4), (40, 0)])
def test_decode_one_long_sequence(window, sinks):
    check_decode(22, 8, 1, 128, [20011], window, sinks)


def test_decode_all_rows_empty():
    check_decode(23, 8, 2, 128, [0, 0, 0], 300, 0, max_len=400)


def test_decode_full_batch_on_a_shared_anchor():
    """Enough sequences on one anchor, all of it in sight: pieces cut at the same places."""
    check_decode(24, 32, 8, 128, [1200 + 13 * i for i in range(64)], 3000, 2, shared=60, rows=[0, 31, 63])


def test_decode_more_sequences_than_a_plan_takes():
    check_decode(25, 4, 1, 64, [(7 * i) % 300 for i in range(1100)], 150, 4, rows=[0, 1, 500, 1099])


def test_decode_loose_bound():
    check_decode(26, 8, 2, 64, [300, 20, 0, 77], 260, 3, max_len=303)


def test_the_last_row_of_a_prefill_is_the_decode():
    """The same operator in its two forms: rows of a prefill against decodes of each length."""
    from paper_2608_14624_amd import ops
    hq, hkv, d, n, rows = 8, 2, 128, 900, 40
    pg = Paged(27, [n], hkv, d)
    q = bf16_bits(pg.rng, rows, hq, d)
    print("[case] prefill rows against decodes", flush=True)
    got, _ = run_prefill(pg, q, [(n - rows, rows)], 200, 6, 0.09)
    lens = np.arange(n - rows + 1, n + 1, dtype=np.int32)
    qd = to_gpu(q)
    out = torch.empty_like(qd)
    ops.cs_decode_window_attn(qd, to_gpu(pg.k), to_gpu(pg.v), to_gpu(np.repeat(pg.tables, rows, 0)), to_gpu(lens),
                              out, max_seq_len=n, window=200, sinks=6, scale=0.09)
    torch.cuda.synchronize()
    ref, mag = window_attention(q, pg.k, pg.v, pg.tables[0], n - rows, hq, hkv, 0.09, 200, 6)
    for x in (got, bf16_bits_to_f64(to_bits(out))):
        assert (np.abs(x - ref) <= attention_bound(ref, mag)).all()
