"""Attention over a pool held in 4 or 8 bits where a wave takes many units of 32 keys in a row, for
every group size, with sequences in any order, and the prefill at scales and queries of all sizes."""

import numpy as np
import pytest

from bounded_cache_util import bf16_bits, to_bits, to_gpu
from oracle import bf16_bits_to_f64, window_attention
from quant_util import QuantPaged, f64, quant_attention_bound
from test_gpu_quant_attention import check_decode, check_prefill, check_rows, run_decode, run_prefill
from test_gpu_quant_range import scaled

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def long_batch(seed, hkv, d, bits, lens, anchor=0, agent=lambda r: 0):
    """Sequences in a pool quantised on the GPU (by the call whose codes are tested one by one), behind
    anchors of `anchor` tokens that the sequences of an agent share: the pool, tables, and the held K and V
    of chosen KV heads for the oracle."""
    from paper_2608_14624_amd import ops
    rng = np.random.default_rng(seed)
    shared = anchor // 16
    own = [-(-n // 16) - shared for n in lens]
    agents = sorted({agent(r) for r in range(len(lens))})
    blocks = shared * len(agents) + sum(own)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    k, v = (torch.randn((blocks, hkv, 16, d), generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    order = rng.permutation(blocks).astype(np.int32)
    anchors = {a: order[i * shared:(i + 1) * shared] for i, a in enumerate(agents)}
    at = shared * len(agents)
    tables = np.zeros((len(lens), shared + max(own)), dtype=np.int32)
    for r, n in enumerate(own):
        tables[r, :shared + n] = np.concatenate([anchors[agent(r)], order[at:at + n]])
        at += n
        if lens[r] % 16:                      # behind the end: NaN
            k[int(tables[r, shared + n - 1]), :, lens[r] % 16:] = float("nan")
            v[int(tables[r, shared + n - 1]), :, lens[r] % 16:] = float("nan")
    ids = torch.arange(blocks, dtype=torch.int32, device="cuda")
    pool = torch.empty(blocks, hkv, ops.kv_quant_tile_bytes(d, bits), dtype=torch.uint8, device="cuda")
    ops.cs_kv_quantize(k, v, ids, ids, pool, bits=bits)
    ops.cs_kv_dequantize(pool, ids, ids, k, v, bits=bits)
    torch.cuda.synchronize()
    return rng, pool, tables, k, v


def decode_long(seed, hq, hkv, d, bits, lens, rows, heads, **kw):
    from paper_2608_14624_amd import ops
    scale = float(np.float32(d ** -0.5))
    rng, pool, tables, k, v = long_batch(seed, hkv, d, bits, lens, **kw)
    q = bf16_bits(rng, len(lens), hq, d)
    out = torch.full((len(lens), hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    ops.cs_decode_quant_attn(to_gpu(q), pool, to_gpu(tables), to_gpu(np.array(lens, dtype=np.int32)), out, bits=bits,
                             max_seq_len=max(lens), scale=scale)
    torch.cuda.synchronize()
    got = bf16_bits_to_f64(to_bits(out))
    assert np.isfinite(got).all()
    for h in heads:
        g = h // (hq // hkv)
        kh, vh = (to_bits(x[:, g:g + 1].contiguous()) for x in (k, v))
        for r in rows:
            ref, mag = window_attention(q[r:r + 1, h:h + 1], kh, vh, tables[r], lens[r] - 1, 1, 1, scale)
            err = np.abs(got[r:r + 1, h:h + 1] - ref)
            assert (err <= quant_attention_bound(ref, mag)).all(), f"sequence {r}, head {h}: {err.max()}"


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
def test_decode_of_long_private_histories(d, bits):
    """Ranges of some 50 units, whose waves refill what they hold several times; the last units are cut
    at every place of their 32 keys."""
    lens = [4225 + 317 * i + (i * 7) % 32 for i in range(14)]
    print(f"[case] 14 long sequences, head_dim {d}, {bits} bits", flush=True)
    units = sum(-(-n // 32) for n in lens)
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    assert units / (2 * cus / 8) > 2 * 4 * 4                # units of a range: twice the four that four waves hold
    decode_long(81, 32, 8, d, bits, lens, rows=range(14), heads=(2, 31))


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("agents", [1, 3])
def test_decode_of_a_batch_in_any_order(d, bits, agents):
    """Sequences on anchors of 2048 tokens, one agent's next to each other or those of several by turns
    (whose blocks are then taken as read once): the same function of the same data."""
    lens = [2048 + 1 + 97 * i for i in range(40)]
    print(f"[case] 40 sequences of {agents} agents by turns, head_dim {d}, {bits} bits", flush=True)
    decode_long(82, 32, 8, d, bits, lens, rows=range(0, 40, 3), heads=(0, 29), anchor=2048, agent=lambda r: r % agents)


@pytest.mark.parametrize("group", [3, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15])
def test_decode_group_sizes(group):
    """With the groups of the other tests (1, 2, 4, 5, 16) every one there is."""
    for d, bits in ((64, 4), (128, 4), (64, 8), (128, 8)):
        check_decode(83, 2 * group, 2, d, bits, [1, 33, 0, 700, 129])


@pytest.mark.parametrize("group", [3, 6, 7, 11, 13, 15, 16])
def test_prefill_group_sizes(group):
    for d, bits in ((64, 4), (128, 8)):
        check_prefill(84, 2 * group, 2, d, bits, [(300, 23), (0, 40), (17, 1)])


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
def test_prefill_large_queries(d, bits):
    """Logits of hundreds: a query's small features count as much as bf16 holds them."""
    scale = float(np.float32(d ** -0.5))
    print(f"[case] large logits, prefill, head_dim {d}, {bits} bits", flush=True)
    invs = [(600, 40), (0, 45)]
    pg = QuantPaged(85, [p + s for p, s in invs], 2, d, bits)
    q = bf16_bits(pg.rng, 85, 8, d)
    q[:, :, ::7] += np.uint16(5 << 7)                     # times 32
    got, cu = run_prefill(pg, q, invs, bits, scale)
    for r, (p, _) in enumerate(invs):
        out, mag = window_attention(q[cu[r]:cu[r + 1]], pg.k, pg.v, pg.tables[r], p, 8, 2, scale)
        # a logit is the sum of 128 products of up to 32 * 4 * 4 that fp32 holds to 2^-24 each: their
        # sum is below 2^12, an error below 128 * 2^-24 * 2^12 * scale = 2^-5 * scale
        bound = quant_attention_bound(out, mag) + 2 * 2.0 ** -5 * scale * mag
        assert (np.abs(got[cu[r]:cu[r + 1]] - out) <= bound).all()


@pytest.mark.parametrize("scale", [0.88, 1.53, 1.0, 2.0, 1e-30])
def test_prefill_scales(scale):
    """Queries of 1/16, so that logits stay of the tests' size; with key parts and without."""
    scale = float(np.float32(scale))
    for bits, d in ((4, 128), (8, 64), (8, 128), (4, 64)):
        for invs in ([(700, 33), (0, 3)], [(10, 300)] * 30):
            print(f"[case] prefill at scale {scale}, head_dim {d}, {bits} bits, {invs[:2]}", flush=True)
            pg = QuantPaged(86, [p + s for p, s in invs], 2, d, bits)
            q = (bf16_bits_to_f64(bf16_bits(pg.rng, sum(s for _, s in invs), 8, d)) / 16).astype(np.float32)
            q = (q.view(np.uint32) >> 16).astype(np.uint16)
            got, cu = run_prefill(pg, q, invs, bits, scale)
            for r in range(2):
                check_rows(got[cu[r]:cu[r + 1]], q[cu[r]:cu[r + 1]], pg, r, invs[r][0], 8, 2, scale)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", ["far below", "tiny"])
def test_small_query_features(case, d, bits):
    """Features 2^15 below the largest of their group of 32 count as bf16 holds them, and so do features
    below 2^-117, next to keys of 2^118, but for what is below 2^-126, which may be lost: a logit then is off by
    2^-126 times the sum of the group's |K|, and a weight and the sum of the weights each by as much."""
    print(f"[case] small query features, {case}, head_dim {d}, {bits} bits", flush=True)
    invs = [(600, 40), (0, 33)]
    pg = QuantPaged(54, [p + s for p, s in invs], 2, d, bits)
    rng = pg.rng
    q, qp = bf16_bits(rng, len(invs), 8, d), bf16_bits(rng, sum(s for _, s in invs), 8, d)
    pg.k[..., :32] = scaled(pg.k[..., :32], 118 if case == "tiny" else 8)
    if case != "tiny":
        pg.k[..., 0] = np.where(pg.k[..., 0] == 0x7FC0, pg.k[..., 0], 0)
    pg.requantise(bits)
    for x in (q, qp):
        small = np.clip(f64(x[..., :32]), -2, 2)
        small = small * (2.0 ** -119 if case == "tiny" else 2.0 ** -10)      # below 2^-117; 2^15 below 64
        x[..., :32] = to_bits(torch.from_numpy(small.astype(np.float32)).bfloat16())
        if case != "tiny":
            x[..., 0] = 0x4280                            # 64
    scale = float(np.float32(d ** -0.5))

    def check(got, q, r, first):
        j = np.arange(first + q.shape[0])
        most = np.abs(f64(pg.k[pg.tables[r, j // 16], :, j % 16, :32])).sum(-1).max()
        out, mag = window_attention(q, pg.k, pg.v, pg.tables[r], first, 8, 2, scale)
        slack = np.expm1(2 * scale * 2.0 ** -126 * most) if case == "tiny" else 0.0
        # (the test tells something only where the bound is far below what the features give)
        assert slack < 0.1
        worst = float((np.abs(got - out) / (quant_attention_bound(out, mag) + slack * (mag + np.abs(out)))).max())
        assert worst <= 1, f"{worst} of the bound"

    got = run_decode(pg, q, bits, scale)
    for r, n in enumerate(pg.lens):
        check(got[r:r + 1], q[r:r + 1], r, int(n) - 1)
    got, cu = run_prefill(pg, qp, invs, bits, scale)
    for r, (p, _) in enumerate(invs):
        check(got[cu[r]:cu[r + 1]], qp[cu[r]:cu[r + 1]], r, p)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
def test_the_largest_query_features(d, bits):
    """Queries of up to 2^128, next to keys of 2^-110: finite, as bf16 is."""
    print(f"[case] the largest query features, head_dim {d}, {bits} bits", flush=True)
    invs = [(600, 40), (0, 33)]
    pg = QuantPaged(56, [p + s for p, s in invs], 2, d, bits)
    rng = pg.rng
    pg.k = scaled(pg.k, -110)
    pg.requantise(bits)
    scale = float(np.float32(d ** -0.5))
    q, qp = (scaled(bf16_bits(rng, n, 8, d), 110) for n in (len(invs), sum(s for _, s in invs)))
    for x in (q, qp):
        x[..., 5], x[..., 40] = 0x7F7F, 0xFF00            # bf16's largest, and -2^127
    for r, n in enumerate(pg.lens):                       # beside keys' zeros
        j = np.arange(n)
        pg.k[pg.tables[r, j // 16], :, j % 16, 5] = 0
        pg.k[pg.tables[r, j // 16], :, j % 16, 40] = 0
    pg.requantise(bits)
    got = run_decode(pg, q, bits, scale)
    for r, n in enumerate(pg.lens):
        check_rows(got[r:r + 1], q[r:r + 1], pg, r, int(n) - 1, 8, 2, scale)
    got, cu = run_prefill(pg, qp, invs, bits, scale)
    for r, (p, _) in enumerate(invs):
        check_rows(got[cu[r]:cu[r + 1]], qp[cu[r]:cu[r + 1]], pg, r, p, 8, 2, scale)
