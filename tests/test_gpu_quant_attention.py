"""Decode and prefill attention over a pool held in 4 or 8 bits against the float64 oracle: lengths
from zero on, every group size, odd batches, with NaN behind every sequence's end and in every block
that none holds."""

import numpy as np
import pytest

from bounded_cache_util import bf16_bits, to_bits, to_gpu
from oracle import bf16_bits_to_f64, window_attention
from quant_util import QuantPaged, quant_attention_bound

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

HEADS = [(8, 2, 128), (4, 4, 64), (5, 1, 128), (16, 1, 64), (6, 3, 128), (40, 8, 64), (16, 1, 128), (32, 8, 128)]


def i32(x):
    return to_gpu(np.asarray(x, dtype=np.int32))


def run_decode(pg, q, bits, scale, max_len=None, workspace="auto", stream=None):
    from paper_2608_14624_amd import ops
    qd = to_gpu(q)
    out = torch.full_like(qd, float("nan"))
    ops.cs_decode_quant_attn(qd, to_gpu(pg.tiles), to_gpu(pg.tables), to_gpu(pg.lens), out, bits=bits,
                             max_seq_len=max_len or max(1, int(pg.lens.max())), scale=scale, workspace=workspace,
                             stream=stream)
    torch.cuda.synchronize()
    return bf16_bits_to_f64(to_bits(out))


def check_rows(got, q, pg, r, pos, hq, hkv, scale, heads=None):
    out, mag = window_attention(q, pg.k, pg.v, pg.tables[r], pos, hq, hkv, scale, heads=heads)
    got = got if heads is None else got[:, list(heads)]
    err = np.abs(got - out)
    assert np.isfinite(err).all(), f"sequence {r}: non-finite output"
    bound = quant_attention_bound(out, mag)
    assert (err <= bound).all(), f"sequence {r}: {err.max()}, {(err / bound).max()} of the bound"


def check_decode(seed, hq, hkv, d, bits, lens, heads=None, seqs=None, room=0, **kw):
    scale = float(np.float32(d ** -0.5))
    print(f"[case] decode {hq}/{hkv} heads of {d}, {bits} bits, {list(lens[:6])}.. ({len(lens)}) {kw}", flush=True)
    pg = QuantPaged(seed, lens, hkv, d, bits, room=room)
    q = bf16_bits(pg.rng, len(lens), hq, d)
    got = run_decode(pg, q, bits, scale, **kw)
    for r, n in enumerate(lens):
        if n == 0:
            assert (got[r] == 0).all(), f"sequence {r}"
        elif seqs is None or r in seqs:
            check_rows(got[r:r + 1], q[r:r + 1], pg, r, n - 1, hq, hkv, scale, heads)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_decode_lengths(hq, hkv, d, bits):
    check_decode(1, hq, hkv, d, bits, [1, 16, 17, 31, 32, 33, 0, 47, 48, 64, 100, 0, 255, 700, 129, 5])


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[1], [2], [9000], [0], [0, 0, 3], [5000, 1, 0, 2047]])
def test_decode_few(d, bits, lens):
    check_decode(2, 8, 2, d, bits, lens)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
def test_decode_many(d, bits):
    """More sequences than a wave counts at once, and more than ranges."""
    rng = np.random.default_rng(3)
    check_decode(3, 4, 1, d, bits, list(rng.integers(0, 90, 700)))
    check_decode(4, 8, 8, d, bits, list(rng.integers(1, 40, 1500)), seqs=range(0, 1500, 37))


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("hq,hkv,d,seqs", [(16, 8, 128, 70), (8, 4, 64, 130)])
def test_decode_on_a_shared_anchor(hq, hkv, d, seqs, bits):
    """Enough sequences on one anchor of 40 blocks that its blocks are asked for and loaded to stay in
    the caches; some end inside it or before its 32nd block, some are empty."""
    rng = np.random.default_rng(7)
    lens = list(rng.integers(640, 1100, seqs - 6)) + [0, 5, 496, 497, 640, 0]
    scale = float(np.float32(d ** -0.5))
    print(f"[case] decode of {seqs} sequences on an anchor, {hq}/{hkv} heads of {d}, {bits} bits", flush=True)
    pg = QuantPaged(7, lens, hkv, d, bits, shared=40)
    q = bf16_bits(pg.rng, len(lens), hq, d)
    got = run_decode(pg, q, bits, scale)
    for r, n in enumerate(lens):
        if n == 0:
            assert (got[r] == 0).all()
        elif r % 7 == 0 or r > seqs - 7:
            check_rows(got[r:r + 1], q[r:r + 1], pg, r, n - 1, hq, hkv, scale)


@pytest.mark.parametrize("bits", [4, 8])
def test_decode_loose_bound_and_workspace(bits):
    """A bound far above the lengths, and a workspace tensor larger than needed."""
    ws = torch.full((1 << 26,), 0xFF, dtype=torch.uint8, device="cuda")      # NaN, were it read
    check_decode(5, 8, 2, 128, bits, [300, 41, 1000], room=20000, max_len=20000, workspace=ws)


def test_decode_workspace_size_is_enforced():
    from paper_2608_14624_amd import ops
    pg = QuantPaged(6, [300, 41], 2, 64, 4)
    q = to_gpu(bf16_bits(pg.rng, 2, 8, 64))
    need = ops.decode_quant_workspace_bytes(2, 300, 8, 2, 64)
    with pytest.raises(ops.CacheScoutError) as e:
        ops.cs_decode_quant_attn(q, to_gpu(pg.tiles), to_gpu(pg.tables), to_gpu(pg.lens), torch.empty_like(q), bits=4,
                                 max_seq_len=300, scale=0.125,
                                 workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    assert e.value.status == ops.CS_ERR_INVALID_ARG


def run_prefill(pg, q, invs, bits, scale, workspace="auto", max_q=None, max_kv=None, stream=None):
    from paper_2608_14624_amd import ops
    cu = np.concatenate([[0], np.cumsum([s for _, s in invs])]).astype(np.int32)
    qd = to_gpu(q)
    out = torch.full_like(qd, float("nan"))
    ops.cs_prefill_quant_attn(
        qd, to_gpu(pg.tiles), to_gpu(pg.tables), i32([p for p, _ in invs]), to_gpu(cu), out, bits=bits,
        max_q_len=max_q or max(s for _, s in invs), max_kv_len=max_kv or max(p + s for p, s in invs), scale=scale,
        workspace=workspace, stream=stream)
    torch.cuda.synchronize()
    return bf16_bits_to_f64(to_bits(out)), cu


def check_prefill(seed, hq, hkv, d, bits, invs, heads=None, **kw):
    scale = float(np.float32(d ** -0.5))
    print(f"[case] prefill {hq}/{hkv} heads of {d}, {bits} bits, {invs[:4]}.. ({len(invs)}) {kw}", flush=True)
    pg = QuantPaged(seed, [p + s for p, s in invs], hkv, d, bits, room=kw.get("max_kv") or 0)
    q = bf16_bits(pg.rng, sum(s for _, s in invs), hq, d)
    got, cu = run_prefill(pg, q, invs, bits, scale, **kw)
    for r, (p, s) in enumerate(invs):
        if s:
            check_rows(got[cu[r]:cu[r + 1]], q[cu[r]:cu[r + 1]], pg, r, p, hq, hkv, scale, heads)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_prefill_ragged(hq, hkv, d, bits):
    check_prefill(11, hq, hkv, d, bits, [(300, 70), (0, 130), (517, 1), (64, 0), (0, 1), (31, 33), (16, 16)],
                  heads=range(min(hq, 8)))


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("invs", [[(0, 1)], [(2000, 1)], [(2100, 20), (1990, 35)], [(5, 3)], [(0, 2), (3000, 2)]])
def test_prefill_key_parts(d, bits, invs):
    check_prefill(12, 8, 2, d, bits, invs)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
def test_prefill_fills_the_device(d, bits):
    """More tiles than the device holds at once: no key parts."""
    check_prefill(13, 32, 8, d, bits, [(700, 1100), (0, 1100), (33, 65), (1, 640)], heads=[0, 13, 31])


@pytest.mark.parametrize("bits", [4, 8])
def test_prefill_more_than_16_heads_per_kv_head(bits):
    check_prefill(14, 24, 1, 64, bits, [(100, 33), (0, 5)])
    check_prefill(15, 34, 2, 128, bits, [(40, 19)])


@pytest.mark.parametrize("bits", [4, 8])
def test_prefill_loose_bounds(bits):
    ws = torch.full((1 << 28,), 0xFF, dtype=torch.uint8, device="cuda")
    check_prefill(16, 8, 2, 128, bits, [(300, 21), (0, 90)], max_q=700, max_kv=9000, workspace=ws)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
def test_large_keys_and_queries(d, bits):
    """Logits of hundreds, where the weights are nearly one key's: a query's small features count
    as much as bf16 holds them."""
    scale = float(np.float32(d ** -0.5))
    print(f"[case] large logits, head_dim {d}, {bits} bits", flush=True)
    pg = QuantPaged(21, [600, 45, 33], 2, d, bits)
    rng = pg.rng
    grow = np.uint16(5 << 7)                                # times 32
    q = bf16_bits(rng, 3, 8, d)
    q[:, :, ::7] += grow
    got = run_decode(pg, q, bits, scale)
    for r, n in enumerate(pg.lens):
        out, mag = window_attention(q[r:r + 1], pg.k, pg.v, pg.tables[r], n - 1, 8, 2, scale)
        # a logit is the sum of 128 products of up to 32 * 4 * 4 that fp32 holds to 2^-24 each: their
        # sum is below 2^12, an error below 128 * 2^-24 * 2^12 * scale = 2^-5 * scale
        slack = 2.0 ** -5 * scale
        bound = quant_attention_bound(out, mag) + 2 * slack * mag
        assert (np.abs(got[r:r + 1] - out) <= bound).all()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
def test_nan_where_the_formula_has_it(d, bits):
    """A query that is not finite makes its own row NaN and no other; so does a NaN key for the rows
    that see it."""
    scale = float(np.float32(d ** -0.5))
    print(f"[case] NaN, head_dim {d}, {bits} bits", flush=True)
    pg = QuantPaged(22, [200, 70, 90], 2, d, bits)
    q = bf16_bits(pg.rng, 3, 8, d)
    q[0, 2, 5], q[1, 7, 40] = 0x7FC0, 0x7F80
    got = run_decode(pg, q, bits, scale)
    bad = np.isnan(got).all(-1)
    want = np.zeros((3, 8), dtype=bool)
    want[0, 2] = want[1, 7] = True
    assert (bad == want).all() and (np.isnan(got).any(-1) == want).all()
