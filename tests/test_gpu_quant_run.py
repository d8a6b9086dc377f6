"""A pool held in 4 or 8 bits as a serving program uses it: together over an anchor's life, captured
and replayed, on other streams, at once, far into a large pool, with logits that rise, and the calls
that are refused."""

import numpy as np
import pytest

from bounded_cache_util import Paged, attention_bound, bf16_bits, to_bits, to_gpu
from oracle import bf16_bits_to_f64, pack_tiles, quantise_rows, row_values, to_bf16_bits, unpack_tiles, window_attention
from quant_util import QuantPaged, quant_attention_bound

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

HQ, HKV = 8, 2


def i32(*x):
    return to_gpu(np.array(x, dtype=np.int32))


def scale_of(d):
    return float(np.float32(d ** -0.5))


def check(got, q, k, v, table, pos, d, bound=quant_attention_bound):
    out, mag = window_attention(q, k, v, table, pos, HQ, HKV, scale_of(d))
    err = np.abs(got - out)
    assert np.isfinite(err).all() and (err <= bound(out, mag)).all(), err.max()


@pytest.mark.parametrize("d,bits", [(128, 4), (64, 8)])
def test_an_anchors_life(d, bits):
    """An anchor that a bf16 prefill left goes cold (to the quantised pool); two invocations hit it
    there, write their suffixes beside it and attend; each decodes some tokens; the anchor returns
    to other blocks of the bf16 pool and a bf16 prefill attends over it."""
    from paper_2608_14624_amd import ops
    print(f"[case] an anchor's life, head_dim {d}, {bits} bits", flush=True)
    anchor, prompts, room = 96, [96 + 75, 96 + 200], 96 + 260
    pg = Paged(31, [room, room], HKV, d, shared=anchor // 16, spare=30)
    rng, kw = pg.rng, dict(bits=bits)
    kd, vd = to_gpu(pg.k), to_gpu(pg.v)
    home = pg.tables[0, :anchor // 16].copy()           # the anchor's blocks in the bf16 pool
    # the quantised pool has its own block ids
    n = pg.num_blocks
    ids = rng.permutation(n)
    tables = ids[pg.tables].astype(np.int32)
    tiles = rng.integers(0, 256, (n, HKV, ops.kv_quant_tile_bytes(d, bits)), dtype=np.uint8)
    pool = to_gpu(tiles)
    ops.cs_kv_quantize(kd, vd, i32(*home), i32(*tables[0, :anchor // 16]), pool, **kw)
    qk, qv = np.full((2, n, HKV, 16, d), 0x7FC0, dtype=np.uint16)
    at = tables[0, :anchor // 16]
    qk[at], qv[at] = (to_bf16_bits(x) for x in unpack_tiles(pack_tiles(pg.k[home], pg.v[home], bits), d, bits))

    def write(tokens, slots):
        k, v = bf16_bits(rng, tokens, HKV, d), bf16_bits(rng, tokens, HKV, d)
        ops.cs_kv_write_quant(to_gpu(k), to_gpu(v), to_gpu(np.array(slots, dtype=np.int32)), pool, **kw)
        for t, s in enumerate(slots):
            qk[s // 16, :, s % 16] = to_bf16_bits(row_values(*quantise_rows(k[t], bits), bits))
            qv[s // 16, :, s % 16] = to_bf16_bits(row_values(*quantise_rows(v[t], bits), bits))

    def slot(r, pos):
        return int(tables[r, pos // 16]) * 16 + pos % 16

    suffix = [p - anchor for p in prompts]
    write(sum(suffix), [slot(r, pos) for r, p in enumerate(prompts) for pos in range(anchor, p)])
    q = bf16_bits(rng, sum(suffix), HQ, d)
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    cu = [0, suffix[0], sum(suffix)]
    td = to_gpu(tables)
    ops.cs_prefill_quant_attn(to_gpu(q), pool, td, i32(anchor, anchor), i32(*cu), out, max_q_len=max(suffix),
                              max_kv_len=max(prompts), scale=scale_of(d), **kw)
    torch.cuda.synchronize()
    got = bf16_bits_to_f64(to_bits(out))
    for r in range(2):
        check(got[cu[r]:cu[r + 1]], q[cu[r]:cu[r + 1]], qk, qv, tables[r], anchor, d)
    lens = list(prompts)
    for _ in range(20):
        write(2, [slot(r, lens[r]) for r in range(2)])
        lens = [x + 1 for x in lens]
        q = bf16_bits(rng, 2, HQ, d)
        out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
        ops.cs_decode_quant_attn(to_gpu(q), pool, td, i32(*lens), out, max_seq_len=room, scale=scale_of(d), **kw)
        torch.cuda.synchronize()
        got = bf16_bits_to_f64(to_bits(out))
        for r in range(2):
            check(got[r:r + 1], q[r:r + 1], qk, qv, tables[r], lens[r] - 1, d)
    # the way back, and the suffix of a new invocation in bf16
    back = np.array(pg.free[:anchor // 16], dtype=np.int32)
    ops.cs_kv_dequantize(pool, i32(*tables[0, :anchor // 16]), to_gpu(back), kd, vd, **kw)
    pg.k[back], pg.v[back] = qk[at], qv[at]
    table = pg.tables[:1].copy()
    table[0, :anchor // 16] = back
    q = bf16_bits(rng, 30, HQ, d)
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    ops.cs_prefill_paged_attn(to_gpu(q), kd, vd, to_gpu(table), i32(anchor), i32(0, 30), out, max_q_len=30,
                              max_kv_len=anchor + 30, scale=scale_of(d))
    torch.cuda.synchronize()
    check(bf16_bits_to_f64(to_bits(out)), q, pg.k, pg.v, table[0], anchor, d, attention_bound)


NAMES = ["write", "quantize", "dequantize", "decode", "prefill"]


def calls(bits=4, d=128):
    """name -> make(**kw) -> (tensors written, run)."""
    from paper_2608_14624_amd import ops
    lens = [700, 33, 0, 260]
    pg = QuantPaged(41, lens, HKV, d, bits, spare=20)
    n, rng = pg.num_blocks, pg.rng
    rows = [40, 33, 0, 21]
    q, qp = to_gpu(bf16_bits(rng, 4, HQ, d)), to_gpu(bf16_bits(rng, sum(rows), HQ, d))
    tiles, t, ld = to_gpu(pg.tiles), to_gpu(pg.tables), to_gpu(pg.lens)
    k, v = to_gpu(bf16_bits(rng, n, HKV, 16, d)), to_gpu(bf16_bits(rng, n, HKV, 16, d))
    slots = to_gpu(rng.permutation(n * 16)[:77].astype(np.int32))
    src, dst = (to_gpu(rng.permutation(n)[:11].astype(np.int32)) for _ in range(2))
    prefix = i32(*[a - b for a, b in zip(lens, rows)])
    cu = to_gpu(np.concatenate([[0], np.cumsum(rows)]).astype(np.int32))

    def write(**kw):
        pool = tiles.clone()
        return [pool], lambda: ops.cs_kv_write_quant(k.view(-1, HKV, d)[:77], v.view(-1, HKV, d)[:77], slots, pool,
                                                     bits=bits, **kw)

    def quantize(**kw):
        pool = tiles.clone()
        return [pool], lambda: ops.cs_kv_quantize(k, v, src, dst, pool, bits=bits, **kw)

    def dequantize(**kw):
        ko, vo = k.clone(), v.clone()
        return [ko, vo], lambda: ops.cs_kv_dequantize(tiles, src, dst, ko, vo, bits=bits, **kw)

    def decode(**kw):
        out = torch.full_like(q, float("nan"))
        return [out], lambda: ops.cs_decode_quant_attn(q, tiles, t, ld, out, bits=bits, max_seq_len=700,
                                                       scale=scale_of(d), **kw)

    def prefill(**kw):
        out = torch.full_like(qp, float("nan"))
        return [out], lambda: ops.cs_prefill_quant_attn(qp, tiles, t, prefix, cu, out, bits=bits, max_q_len=40,
                                                        max_kv_len=700, scale=scale_of(d), **kw)

    return dict(zip(NAMES, (write, quantize, dequantize, decode, prefill)))


def same(a, b):
    return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


@pytest.mark.parametrize("name", NAMES)
def test_captured_and_replayed(name):
    """Several replays, eager work between them, equal the eager call."""
    make = calls()[name]
    print(f"[case] {name} captured", flush=True)
    eager, run_eager = make()
    run_eager()
    written, run = make()
    start = [x.clone() for x in written]
    run()
    for x, y in zip(written, start):
        x.copy_(y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    torch.cuda.synchronize()
    for _ in range(4):
        for x, y in zip(written, start):
            x.copy_(y)
        graph.replay()
        run_eager()
        torch.cuda.synchronize()
        assert same(written, eager)


def test_replays_follow_the_lengths():
    """A captured write and decode of a batch that grows: lengths, slots and rows change in place."""
    from paper_2608_14624_amd import ops
    d, bits, room = 128, 4, 400
    print("[case] a captured decode step that grows", flush=True)
    pg = QuantPaged(42, [room, room], HKV, d, bits)
    pool, td = to_gpu(pg.tiles), to_gpu(pg.tables)
    rng = pg.rng
    k, v, q = (torch.zeros(2, h, d, dtype=torch.bfloat16, device="cuda") for h in (HKV, HKV, HQ))
    slots, lens, out = i32(0, 0), i32(1, 1), torch.zeros_like(q)

    def step():
        ops.cs_kv_write_quant(k, v, slots, pool, bits=bits)
        ops.cs_decode_quant_attn(q, pool, td, lens, out, bits=bits, max_seq_len=room, scale=scale_of(d))

    slots.fill_(-1)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in ([1, 17], [2, 0], [33, 255], [399, 64]):
        kn, vn, qn = bf16_bits(rng, 2, HKV, d), bf16_bits(rng, 2, HKV, d), bf16_bits(rng, 2, HQ, d)
        at = [int(pg.tables[r, (x - 1) // 16]) * 16 + (x - 1) % 16 if x else -1 for r, x in enumerate(n)]
        for dst, x in ((k, kn), (v, vn), (q, qn)):
            dst.copy_(to_gpu(x))
        slots.copy_(i32(*at))
        lens.copy_(i32(*n))
        graph.replay()
        torch.cuda.synchronize()
        for r, x in enumerate(n):
            if x:
                b, o = at[r] // 16, at[r] % 16
                pg.k[b, :, o] = to_bf16_bits(row_values(*quantise_rows(kn[r], bits), bits))
                pg.v[b, :, o] = to_bf16_bits(row_values(*quantise_rows(vn[r], bits), bits))
        got = bf16_bits_to_f64(to_bits(out))
        for r, x in enumerate(n):
            if x:
                check(got[r:r + 1], qn[r:r + 1], pg.k, pg.v, pg.tables[r], x - 1, d)
            else:
                assert (got[r] == 0).all()


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("how", ["stream", "handle", "current"])
def test_other_streams(name, how):
    make = calls()[name]
    print(f"[case] {name} on a side stream ({how})", flush=True)
    want, run = make()
    run()
    side = torch.cuda.Stream()
    got, run = make(**({} if how == "current" else {"stream": side if how == "stream" else side.cuda_stream}))
    torch.cuda.synchronize()
    if how == "current":
        with torch.cuda.stream(side):
            run()
    else:
        run()
    torch.cuda.synchronize()
    assert same(got, want)


@pytest.mark.parametrize("bits,d", [(4, 128), (8, 64)])
def test_all_at_once(bits, d):
    """Every operator twice, on streams of their own, with nothing between them."""
    made = calls(bits, d)
    print(f"[case] all operators at once, {bits} bits", flush=True)
    want = {}
    for name in NAMES:
        want[name], run = made[name]()
        run()
    torch.cuda.synchronize()
    got = [(name, *made[name](stream=torch.cuda.Stream())) for name in NAMES * 2]
    torch.cuda.synchronize()
    for _, _, run in got:
        run()
    torch.cuda.synchronize()
    for name, written, _ in got:
        assert same(written, want[name]), name


@pytest.mark.parametrize("bits", [4, 8])
def test_blocks_past_two_to_the_32_bytes(bits):
    """The same blocks at the end of a pool of more than 2^32 bytes: the same results, bit for bit."""
    from paper_2608_14624_amd import ops
    hkv, hq, d = 8, 32, 128
    size = ops.kv_quant_tile_bytes(d, bits)
    lens = [700, 1500]
    pg = QuantPaged(43, lens, hkv, d, bits, spare=10)
    n = pg.num_blocks
    far = (1 << 32) // (hkv * size) + n + 7
    q, qp = to_gpu(bf16_bits(pg.rng, 2, hq, d)), to_gpu(bf16_bits(pg.rng, 150, hq, d))
    k, v = to_gpu(bf16_bits(pg.rng, n, hkv, 16, d)), to_gpu(bf16_bits(pg.rng, n, hkv, 16, d))
    ids = to_gpu(pg.rng.permutation(n)[:9].astype(np.int32))
    slots = to_gpu(pg.rng.permutation(16 * n)[:50].astype(np.int32))
    print(f"[case] a pool of {far * hkv * size} bytes", flush=True)
    results = []
    for offset in (0, far - n):
        pool = torch.empty(n + offset, hkv, size, dtype=torch.uint8, device="cuda")
        pool[offset:] = to_gpu(pg.tiles)
        t = to_gpu(pg.tables + np.int32(offset))
        out, outp, kb, vb = torch.empty_like(q), torch.empty_like(qp), k.clone(), v.clone()
        ops.cs_decode_quant_attn(q, pool, t, to_gpu(pg.lens), out, bits=bits, max_seq_len=1500, scale=scale_of(d))
        ops.cs_prefill_quant_attn(qp, pool, t, i32(650, 1400), i32(0, 50, 150), outp, bits=bits, max_q_len=100,
                                  max_kv_len=1500, scale=scale_of(d))
        ops.cs_kv_write_quant(k.view(-1, hkv, d)[:50], v.view(-1, hkv, d)[:50], slots + 16 * offset, pool, bits=bits)
        ops.cs_kv_quantize(k, v, ids, ids + offset, pool, bits=bits)
        ops.cs_kv_dequantize(pool, ids.flip(0).contiguous() + offset, ids, kb, vb, bits=bits)
        torch.cuda.synchronize()
        results.append([x.clone() for x in (out, outp, kb, vb, pool[offset:])])
        del pool
    assert same(*results)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rise", [280.0, -280.0])
def test_rising_and_falling_logits(d, bits, rise):
    """Logits that change by hundreds along the keys, so that the softmax's reference has to move
    many times or never again; decode and prefill.  (An exponent of up to 600 carries 16 roundings
    of 2^-24 of itself, 6e-4, once in a weight and once in the sum.)"""
    print(f"[case] logits that change by {rise}, head_dim {d}, {bits} bits", flush=True)
    n, rows = 1100, 40
    pg = Paged(44, [n], HKV, d)
    k = bf16_bits_to_f64(pg.k).astype(np.float32)
    for j in range(n):                     # every query's first feature is 16
        k[pg.tables[0, j // 16], :, j % 16, 0] = rise * j / n
    q = bf16_bits_to_f64(bf16_bits(pg.rng, rows, HQ, d))
    q[:, :, 0] = 16.0
    q = to_bits(to_gpu(q.astype(np.float32)).bfloat16())
    pg.k[:] = to_bits(to_gpu(k).bfloat16())
    pg.k[pg.tables[0, n // 16], :, n % 16:] = 0x7FC0
    QuantPaged.requantise(pg, bits)
    from paper_2608_14624_amd import ops
    out = torch.empty(rows, HQ, d, dtype=torch.bfloat16, device="cuda")
    one = torch.empty(1, HQ, d, dtype=torch.bfloat16, device="cuda")
    ops.cs_prefill_quant_attn(to_gpu(q), to_gpu(pg.tiles), to_gpu(pg.tables), i32(n - rows), i32(0, rows), out,
                              bits=bits, max_q_len=rows, max_kv_len=n, scale=scale_of(d))
    ops.cs_decode_quant_attn(to_gpu(q[-1:]), to_gpu(pg.tiles), to_gpu(pg.tables), i32(n), one, bits=bits, max_seq_len=n,
                             scale=scale_of(d))
    torch.cuda.synchronize()

    def bound(out, mag):
        return quant_attention_bound(out, mag) + 1.2e-3 * mag

    check(bf16_bits_to_f64(to_bits(out)), q, pg.k, pg.v, pg.tables[0], n - rows, d, bound)
    check(bf16_bits_to_f64(to_bits(one)), q[-1:], pg.k, pg.v, pg.tables[0], n - 1, d, bound)


@pytest.mark.parametrize("scale", [0.88, 1.53, 1.0, 2.0, 1e-30, 40.0])
def test_scales(scale):
    """Scales from tiny to large (queries of 1/16, so that logits stay of the tests' size up to 2; at 40
    the exponents are 20 times as large, and so are their roundings)."""
    from paper_2608_14624_amd import ops
    print(f"[case] scale {scale}", flush=True)
    scale = float(np.float32(scale))
    for bits, d in ((4, 128), (8, 64)):
        pg = QuantPaged(45, [700, 3, 45], HKV, d, bits)
        q = (bf16_bits_to_f64(bf16_bits(pg.rng, 3, HQ, d)) / 16).astype(np.float32)
        q = (q.view(np.uint32) >> 16).astype(np.uint16)
        out = torch.empty(3, HQ, d, dtype=torch.bfloat16, device="cuda")
        ops.cs_decode_quant_attn(to_gpu(q), to_gpu(pg.tiles), to_gpu(pg.tables), to_gpu(pg.lens), out, bits=bits,
                                 max_seq_len=700, scale=scale)
        torch.cuda.synchronize()
        got = bf16_bits_to_f64(to_bits(out))
        for r, n in enumerate(pg.lens):
            ref, mag = window_attention(q[r:r + 1], pg.k, pg.v, pg.tables[r], n - 1, HQ, HKV, scale)
            bound = quant_attention_bound(ref, mag) + (8e-3 * mag if scale > 2 else 0)
            assert (np.abs(got[r:r + 1] - ref) <= bound).all()


def test_results_do_not_change_from_run_to_run():
    for bits in (4, 8):
        made = calls(bits)
        for name in NAMES:
            print(f"[case] {name} twice, {bits} bits", flush=True)
            results = []
            for _ in range(3):
                written, run = made[name]()
                run()
                torch.cuda.synchronize()
                results.append(written)
            assert same(results[0], results[1]) and same(results[0], results[2])


def test_wrong_tensors_are_refused():
    from paper_2608_14624_amd import ops
    d, bits = 128, 4
    pg = QuantPaged(46, [50, 20], HKV, d, bits)
    tiles, t, ld = to_gpu(pg.tiles), to_gpu(pg.tables), to_gpu(pg.lens)
    q = to_gpu(bf16_bits(pg.rng, 2, HQ, d))
    k, v = to_gpu(pg.k), to_gpu(pg.v)
    ids, slots = i32(0, 1), i32(3, 4)
    new = to_gpu(bf16_bits(pg.rng, 2, HKV, d))

    def decode(q=q, pool=tiles, t=t, ld=ld, out=None, bits=bits, **kw):
        return ops.cs_decode_quant_attn(q, pool, t, ld, torch.empty_like(q) if out is None else out, bits=bits,
                                        max_seq_len=50, scale=0.1, **kw)

    def prefill(q=q, pool=tiles, cu=i32(0, 1, 2), p=i32(4, 5), **kw):
        return ops.cs_prefill_quant_attn(q, pool, t, p, cu, torch.empty_like(q), max_q_len=1, max_kv_len=50, scale=0.1,
                                         **{"bits": bits, **kw})

    def write(k=new, v=new, slots=slots, pool=tiles, bits=bits):
        return ops.cs_kv_write_quant(k, v, slots, pool, bits=bits)

    def quantize(k=k, v=v, a=ids, b=ids, pool=tiles, bits=bits):
        return ops.cs_kv_quantize(k, v, a, b, pool, bits=bits)

    def dequantize(k=k, v=v, a=ids, b=ids, pool=tiles, bits=bits):
        return ops.cs_kv_dequantize(pool, a, b, k, v, bits=bits)

    other = torch.zeros(tiles.shape[0], HKV, ops.kv_quant_tile_bytes(64, 4), dtype=torch.uint8, device="cuda")
    for call in (decode, prefill, write, quantize, dequantize):
        for bad in (dict(pool=other), dict(pool=tiles.float()), dict(pool=tiles.cpu()), dict(pool=tiles[:, :, :-1]),
                    dict(bits=8), dict(bits=3), dict(pool=tiles.view(-1))):
            with pytest.raises(ops.CacheScoutError):
                call(**bad)
    one = tiles[:, :1].contiguous()
    for call, bad in ((write, dict(pool=one)), (quantize, dict(pool=one)), (dequantize, dict(pool=one)),
                      (decode, dict(q=q.float())), (decode, dict(q=q[0])), (decode, dict(t=t.long())),
                      (decode, dict(ld=ld[:1])), (decode, dict(out=q[:1])), (decode, dict(workspace=None)),
                      (prefill, dict(cu=i32(0, 2))), (prefill, dict(p=i32(4))), (write, dict(k=new[:1])),
                      (write, dict(slots=slots[:1])), (write, dict(k=new.half())), (quantize, dict(a=ids[:1])),
                      (quantize, dict(v=v[:-1])), (dequantize, dict(b=ids.long())), (dequantize, dict(k=k[:, :1]))):
        with pytest.raises(ops.CacheScoutError):
            call(**bad)


def test_debug_checks_refuse_bad_metadata(monkeypatch):
    from paper_2608_14624_amd import ops
    monkeypatch.setenv("CS_DEBUG_CHECK", "1")
    d, bits = 64, 8
    pg = QuantPaged(47, [50, 20], HKV, d, bits)
    n = pg.num_blocks
    tiles, k, v = to_gpu(pg.tiles), to_gpu(pg.k), to_gpu(pg.v)
    q = to_gpu(bf16_bits(pg.rng, 2, HQ, d))
    new = to_gpu(bf16_bits(pg.rng, 2, HKV, d))
    bad_table = pg.tables.copy()
    bad_table[0, 1] = n

    def decode(lens, table=pg.tables):
        return lambda: ops.cs_decode_quant_attn(q, tiles, to_gpu(table), i32(*lens), torch.empty_like(q), bits=bits,
                                                max_seq_len=50, scale=0.1)

    def prefill(prefix, cu, table=pg.tables):
        return lambda: ops.cs_prefill_quant_attn(q, tiles, to_gpu(table), i32(*prefix), i32(*cu), torch.empty_like(q),
                                                 bits=bits, max_q_len=1, max_kv_len=50, scale=0.1)

    def write(*slots):
        return lambda: ops.cs_kv_write_quant(new, new, i32(*slots), tiles, bits=bits)

    def quantize(src, dst):
        return lambda: ops.cs_kv_quantize(k, v, i32(*src), i32(*dst), tiles, bits=bits)

    def dequantize(src, dst):
        return lambda: ops.cs_kv_dequantize(tiles, i32(*src), i32(*dst), k, v, bits=bits)

    for good in (decode([50, 0]), prefill([49, 19], [0, 1, 2]), write(3, -1), quantize([1, 1], [0, 2]),
                 dequantize([1, 1], [0, 2])):
        good()
    for bad in (decode([51, 20]), decode([50, -1]), decode([50, 20], bad_table), prefill([50, 19], [0, 1, 2]),
                prefill([49, -1], [0, 1, 2]), prefill([49, 19], [0, 1, 1]), prefill([49, 19], [0, 1, 2], bad_table),
                write(16 * n, 0), write(4, 4), quantize([0, n], [0, 1]), quantize([0, 1], [1, 1]),
                quantize([0, 1], [0, -1]), dequantize([0, -1], [0, 1]), dequantize([0, 1], [2, 2]),
                dequantize([0, 1], [0, n])):
        with pytest.raises(ops.CacheScoutError) as e:
            bad()
        assert e.value.status == ops.CS_ERR_INVALID_ARG
    torch.cuda.synchronize()
