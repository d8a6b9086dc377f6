"""Scales from ln 2 on, where the softmax's first reference, a lowest value divided by the scale and
multiplied by it again, has to stay finite: rows that see none of the first keys."""

import numpy as np
import pytest

from bounded_cache_util import Paged, attention_bound, bf16_bits, to_bits, to_gpu, weight_bound
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


def minus_infinity(pg, q, r, first, below):
    """The 32 keys from `first` on of sequence r get a feature of -inf, and in `below` one whose logits,
    with a query feature of 1, weigh nothing in float64 either."""
    q[:, :, 0] = 0x3F80
    for b in (first // 16, first // 16 + 1):
        pg.k[pg.tables[r, b], :, :, 0] = 0xFF80
        below[pg.tables[r, b], :, :, 0] = 0xC8C3           # -399,360


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,lens", [(32, 8, [3000, 700] + [90] * 14), (8, 2, [620 + 7 * i for i in range(130)])])
def test_decode_with_logits_of_minus_infinity(scale, d, hq, hkv, lens):
    """Units of 32 keys whose logits are all -inf, at the start of a range and inside one, in the
    decodes in ranges and by pairs: they weigh nothing."""
    from paper_2608_14624_amd import ops
    scale, n_seqs = float(np.float32(scale)), len(lens)
    print(f"[case] decode of -inf logits at scale {scale}, heads of {d}, {n_seqs} sequences", flush=True)
    pg = Paged(73, lens, hkv, d, room=14000 if n_seqs == 16 else 0)
    q = small_queries(pg.rng, n_seqs, hq, d)
    below = pg.k.copy()
    for r, first in ((0, 0), (0, 64), (0, 128), (0, 512), (1, 160)):
        minus_infinity(pg, q, r, first, below)
    qd, kd, vd, td, ld = to_gpu(q), to_gpu(pg.k), to_gpu(pg.v), to_gpu(pg.tables), to_gpu(pg.lens)
    zero = torch.zeros(n_seqs, dtype=torch.int32, device="cuda")
    sd = torch.zeros(pg.num_blocks, hkv, 16, device="cuda")
    outs = {name: torch.full_like(qd, float("nan")) for name in ("plain", "window", "scored")}
    ops.cs_paged_decode_attn(qd, kd, vd, td, ld, outs["plain"], max_seq_len=max(lens), scale=scale)
    ops.cs_decode_window_attn(qd, kd, vd, td, ld, outs["window"], max_seq_len=max(lens), window=max(lens), sinks=0,
                              scale=scale)
    ops.cs_decode_attn_scores(qd, kd, vd, td, ld, zero, sd, outs["scored"], max_seq_len=max(lens),
                              max_scored_len=max(lens), scale=scale)
    if n_seqs == 16 and d == 128:          # the bounds of a cascade in ranges
        outs["cascade"] = torch.full_like(qd, float("nan"))
        groups = torch.arange(0, 17, 4, dtype=torch.int32, device="cuda")
        ops.cs_cascade_decode_attn(qd, kd, vd, td, ld, groups, zero[:4].contiguous(), outs["cascade"], max_seq_len=14000,
                                   max_group_seqs=4, max_shared_len=10000, max_rest_len=4000, scale=scale)
    torch.cuda.synchronize()
    want, got = np.zeros((pg.num_blocks, hkv, 16)), sd.cpu().numpy()
    for r in (0, 1):
        n = lens[r]
        ref, mag = window_attention(q[r:r + 1], below, pg.v, pg.tables[r], n - 1, hq, hkv, scale)
        for name, out in outs.items():
            err = np.abs(bf16_bits_to_f64(to_bits(out[r:r + 1])) - ref)
            assert np.isfinite(err).all(), f"{name}, sequence {r}: not finite"
            assert (err <= attention_bound(ref, mag)).all(), f"{name}, sequence {r}: {err.max()}"
        add_key_scores(want, q[r:r + 1], below, pg.tables[r], n - 1, n - 1, 0, hq, hkv, scale, 1.0)
        j = np.arange(n)
        at = pg.tables[r, j // 16], slice(None), j % 16
        assert np.isfinite(got[at]).all(), f"sequence {r}: scores are not finite"
        assert (np.abs(got[at] - want[at]) <= weight_bound(want[at])).all(), f"scores of sequence {r}"
