"""Scales from ln 2 on, where the softmax's first reference, a lowest value divided by the scale and
multiplied by it again, has to stay finite: rows that see none of the first keys."""

import numpy as np
import pytest

from bounded_cache_util import Paged, attention_bound, bf16_bits, to_gpu, weight_bound
from oracle import add_key_scores, bf16_bits_to_f64, window_attention
from test_gpu_window_attention import prefill_batch, run_prefill

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# The largest float32 divided by scale / ln 2 and multiplied by it again is infinite for the first two.
SCALES = [0.88, 1.53, 1.0, 2.0]


def small_queries(rng, *shape):
    """N(0, 1) / 16 as bf16 bits, exactly: logits of the size that N(0, 1) queries have at scales of a
    tenth, so that the tests' error bounds hold."""
    x = (bf16_bits_to_f64(bf16_bits(rng, *shape)) / 16).astype(np.float32)
    return (x.view(np.uint32) >> 16).astype(np.uint16)


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64)])
@pytest.mark.parametrize("invs,rows", [([(0, 130), (0, 1), (0, 5)], 130), ([(4000, 40), (0, 500)], 40),
                                       ([(0, 2500)], 2500)])
def test_prompt_scores(scale, hq, hkv, d, invs, rows):
    """Rows at the first positions, where half a wave's lanes hold no visible key, and key parts of
    which the earlier rows see nothing."""
    from paper_2608_14624_amd import ops
    scale = float(np.float32(scale))
    print(f"[case] prompt scores at scale {scale}, {hq}/{hkv} heads of {d}, {invs}, rows {rows}", flush=True)
    pg = Paged(71, [p + s for p, s in invs], hkv, d)
    q = small_queries(pg.rng, sum(s for _, s in invs), hq, d)
    cu = np.concatenate([[0], np.cumsum([s for _, s in invs])]).astype(np.int32)
    sd = to_gpu(np.zeros((pg.num_blocks, hkv, 16), dtype=np.float32))
    ops.cs_prefill_key_scores(to_gpu(q), to_gpu(pg.k), to_gpu(pg.tables),
                              to_gpu(np.array([p for p, _ in invs], dtype=np.int32)), to_gpu(cu),
                              to_gpu(np.zeros(len(invs), dtype=np.int32)), sd, max_q_len=max(s for _, s in invs),
                              max_kv_len=max(p + s for p, s in invs), rows=rows, scale=scale)
    torch.cuda.synchronize()
    got, want = sd.cpu().numpy(), np.zeros((pg.num_blocks, hkv, 16))
    for r, (p, s) in enumerate(invs):
        n = min(s, rows)
        add_key_scores(want, q[cu[r + 1] - n:cu[r + 1]], pg.k, pg.tables[r], p + s - n, p, 0, hq, hkv, scale, 1.0)
    assert np.isfinite(got).all(), f"{(~np.isfinite(got)).sum()} scores are not finite"
    assert (np.abs(got - want) <= weight_bound(want)).all(), np.abs(got - want).max()


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("invs", [[(700, 1100), (0, 1100)],
                                  [(500, 900), (0, 1300), (80, 3), (0, 0), (1200, 700), (33, 65), (0, 640)],
                                  [(300, 70), (0, 130), (517, 1)]])
@pytest.mark.parametrize("window,sinks", [(1, 0), (37, 9)])
def test_window_prefill(scale, d, invs, window, sinks):
    """Equal and ragged ping-pong tiles and split tiles under a window that leaves a tile's later rows
    nothing of its first step."""
    scale, hq, hkv, heads = float(np.float32(scale)), 32, 8, [5, 30]
    print(f"[case] window prefill at scale {scale}, heads of {d}, {invs}, window {window}, sinks {sinks}", flush=True)
    pg, _ = prefill_batch(72, hq, hkv, d, invs, window, sinks)
    q = small_queries(pg.rng, sum(s for _, s in invs), hq, d)
    got, cu = run_prefill(pg, q, invs, window, sinks, scale)
    for r, (p, s) in enumerate(invs):
        if s == 0:
            continue
        out, mag = window_attention(q[cu[r]:cu[r + 1]], pg.k, pg.v, pg.tables[r], p, hq, hkv, scale, window, sinks,
                                    heads)
        err = np.abs(got[cu[r]:cu[r + 1]][:, heads] - out)
        assert np.isfinite(err).all(), f"invocation {r}: {(~np.isfinite(err)).sum()} elements are not finite"
        assert (err <= attention_bound(out, mag)).all(), f"invocation {r}: {err.max()}"
