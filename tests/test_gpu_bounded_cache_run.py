"""The operators that bound a cache as a serving program uses them: together over a sequence's
life, captured and replayed, on other streams, at once, with pools past 2^31 elements, and the calls
that are refused."""

import numpy as np
import pytest

from bounded_cache_util import Paged, attention_bound, bf16_bits, to_bits, to_gpu, weight_bound
from oracle import add_key_scores, bf16_bits_to_f64, evict, window_attention

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

HQ, HKV, D = 8, 2, 128
SCALE = float(np.float32(D ** -0.5))


def i32(*x):
    return to_gpu(np.array(x, dtype=np.int32))


def test_a_sequences_life():
    """Two agents' sequences on one anchor: a prefill under a window, the prompt's scores, decode
    steps that write their token and add its weights, an eviction within the sequences' blocks, more
    steps, an eviction into new blocks, a last step; every output and score against the oracle, every
    choice exact for the scores that it was made from."""
    from paper_2608_14624_amd import ops
    anchor, prompts, room = 64, [300, 170], 420
    pg = Paged(61, [room, room], HKV, D, shared=anchor // 16, spare=40)
    rng = pg.rng
    tables, froms = pg.tables.copy(), np.array([anchor, anchor], dtype=np.int32)
    k, v = pg.k.copy(), pg.v.copy()
    scores = rng.random((pg.num_blocks, HKV, 16)).astype(np.float32)
    kd, vd, sd, fd = to_gpu(k), to_gpu(v), to_gpu(scores), to_gpu(froms)

    # prompts: their K and V, attention under a window, scores of the last 50 rows
    suffix = [p - anchor for p in prompts]
    kn, vn = (bf16_bits(rng, sum(suffix), HKV, D) for _ in range(2))
    slots = np.concatenate([tables[r, np.arange(anchor, p) // 16] * 16 + np.arange(anchor, p) % 16
                            for r, p in enumerate(prompts)]).astype(np.int32)
    ops.cs_kv_write(to_gpu(kn), to_gpu(vn), to_gpu(slots), kd, vd)
    k[slots // 16, :, slots % 16], v[slots // 16, :, slots % 16] = kn, vn
    q = bf16_bits(rng, sum(suffix), HQ, D)
    cu = [0, suffix[0], sum(suffix)]
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    ops.cs_prefill_window_attn(to_gpu(q), kd, vd, to_gpu(tables), fd, i32(*cu), out, max_q_len=max(suffix),
                               max_kv_len=max(prompts), window=90, sinks=4, scale=SCALE)
    ops.cs_prefill_key_scores(to_gpu(q), kd, to_gpu(tables), fd, i32(*cu), fd, sd, max_q_len=max(suffix),
                              max_kv_len=max(prompts), rows=50, scale=SCALE)
    torch.cuda.synchronize()
    got, want = bf16_bits_to_f64(to_bits(out)), scores.astype(np.float64)
    for r, p in enumerate(prompts):
        rows = q[cu[r]:cu[r + 1]]
        ref, mag = window_attention(rows, k, v, tables[r], anchor, HQ, HKV, SCALE, 90, 4)
        assert (np.abs(got[cu[r]:cu[r + 1]] - ref) <= attention_bound(ref, mag)).all()
        add_key_scores(want, rows[-50:], k, tables[r], p - 50, anchor, anchor, HQ, HKV, SCALE, 1.0)
    lens = np.array(prompts, dtype=np.int32)
    check_scores(sd, want, tables, lens, anchor)

    def steps(n):
        nonlocal lens, want
        for _ in range(n):
            lens = lens + 1
            kn, vn, q = bf16_bits(rng, 2, HKV, D), bf16_bits(rng, 2, HKV, D), bf16_bits(rng, 2, HQ, D)
            at = tables[[0, 1], (lens - 1) // 16], (lens - 1) % 16
            ops.cs_kv_write(to_gpu(kn), to_gpu(vn), to_gpu((at[0] * 16 + at[1]).astype(np.int32)), kd, vd)
            k[at[0], :, at[1]], v[at[0], :, at[1]] = kn, vn
            out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
            want = sd.cpu().numpy().astype(np.float64)
            ops.cs_decode_attn_scores(to_gpu(q), kd, vd, to_gpu(tables), to_gpu(lens), fd, sd, out, max_seq_len=room,
                                      max_scored_len=room - anchor, scale=SCALE, decay=0.9)
            torch.cuda.synchronize()
            got = bf16_bits_to_f64(to_bits(out))
            for r, n_keys in enumerate(lens):
                ref, mag = window_attention(q[r:r + 1], k, v, tables[r], n_keys - 1, HQ, HKV, SCALE)
                assert (np.abs(got[r:r + 1] - ref) <= attention_bound(ref, mag)).all()
                add_key_scores(want, q[r:r + 1], k, tables[r], n_keys - 1, n_keys - 1, anchor, HQ, HKV, SCALE,
                               float(np.float32(0.9)))
            check_scores(sd, want, tables, lens, anchor)

    def shrink(dst, budget, trigger, recent):
        nonlocal lens, tables
        s = sd.cpu().numpy()
        kept = torch.empty(2, HKV, budget, dtype=torch.int32, device="cuda")
        ld = to_gpu(lens)
        ops.cs_kv_evict(sd, kd, vd, to_gpu(tables), None if dst is None else to_gpu(dst), ld, fd, kept, ld,
                        max_seq_len=room, budget=budget, trigger=trigger, recent=recent)
        torch.cuda.synchronize()
        moved = []
        for r in range(2):
            got, n = evict(s, k, v, tables[r], None if dst is None else dst[r], int(lens[r]), anchor, budget, trigger,
                           recent)
            moved.append(got is not None)
            assert int(kept[r, 0, 0]) == (-1 if got is None else got[0][0])
            assert got is None or (kept[r].cpu().numpy() == got).all()
            lens[r] = n
        assert (ld.cpu().numpy() == lens).all()
        assert (to_bits(kd) == k).all() and (to_bits(vd) == v).all()
        assert (sd.cpu().numpy() == s).all()
        if dst is not None:
            tables = np.where(np.array(moved)[:, None], dst, tables)
        return moved

    print("[case] a sequence's life", flush=True)
    steps(5)
    assert shrink(None, 100, 200, 16) == [True, False]
    steps(20)
    dst = tables.copy()
    for r in range(2):
        dst[r, anchor // 16:anchor // 16 + 6] = pg.free[10 * r:10 * r + 6]
    assert shrink(dst, 90, 110, 30) == [True, True]
    steps(2)


def check_scores(sd, want, tables, lens, first):
    got = sd.cpu().numpy()
    for r, n in enumerate(lens):
        j = np.arange(first, n)
        at = tables[r, j // 16], slice(None), j % 16
        assert (np.abs(got[at] - want[at]) <= weight_bound(want[at])).all()


def calls():
    """Each operator on inputs of its own: (what it writes, a function that makes it run)."""
    from paper_2608_14624_amd import ops
    lens, width = [1300, 77, 0, 333], 84
    pg = Paged(62, lens, HKV, D, spare=60)
    kd, vd, td = to_gpu(pg.k), to_gpu(pg.v), to_gpu(pg.tables[:, :width].copy())
    ld, qd = to_gpu(pg.lens), to_gpu(bf16_bits(pg.rng, 4, HQ, D))
    scores = to_gpu(pg.rng.random((pg.num_blocks, HKV, 16)).astype(np.float32))
    zero = i32(0, 0, 0, 0)
    cu, prefix = i32(0, 60, 137, 137, 237), i32(1240, 0, 0, 233)
    qp = to_gpu(bf16_bits(pg.rng, 237, HQ, D))
    dst = pg.tables[:, :width].copy()
    dst[0, :20], dst[3, :20] = pg.free[:20], pg.free[20:40]
    dd = to_gpu(dst)

    def window_decode(**kw):
        out = torch.empty_like(qd)
        return [out], lambda: ops.cs_decode_window_attn(qd, kd, vd, td, ld, out, max_seq_len=1300, window=300, sinks=5,
                                                        scale=SCALE, **kw)

    def window_prefill(**kw):
        out = torch.empty_like(qp)
        return [out], lambda: ops.cs_prefill_window_attn(qp, kd, vd, td, prefix, cu, out, max_q_len=100,
                                                         max_kv_len=1300, window=1000, sinks=5, scale=SCALE, **kw)

    def decode_scores(**kw):
        out, s = torch.empty_like(qd), scores.clone()
        return [out, s], lambda: ops.cs_decode_attn_scores(qd, kd, vd, td, ld, zero, s, out, max_seq_len=1300,
                                                           max_scored_len=1300, scale=SCALE, decay=0.5, **kw)

    def prefill_scores(**kw):
        s = scores.clone()
        return [s], lambda: ops.cs_prefill_key_scores(qp, kd, td, prefix, cu, zero, s, max_q_len=100, max_kv_len=1300,
                                                      rows=80, scale=SCALE, decay=0.5, **kw)

    def evict_to_other_blocks(**kw):
        k, v, s = kd.clone(), vd.clone(), scores.clone()
        kept, new = torch.zeros(4, HKV, 200, dtype=torch.int32, device="cuda"), torch.zeros_like(ld)
        return [k, v, s, kept, new], lambda: ops.cs_kv_evict(s, k, v, td, dd, ld, zero, kept, new, max_seq_len=1300,
                                                             budget=200, trigger=250, recent=20, **kw)

    def evict_in_place(**kw):
        k, v, s = kd.clone(), vd.clone(), scores.clone()
        kept, new = torch.zeros(4, HKV, 200, dtype=torch.int32, device="cuda"), torch.zeros_like(ld)
        return [k, v, s, kept, new], lambda: ops.cs_kv_evict(s, k, v, td, None, ld, zero, kept, new, max_seq_len=1300,
                                                             budget=200, trigger=250, recent=20, **kw)

    return dict(window_decode=window_decode, window_prefill=window_prefill, decode_scores=decode_scores,
                prefill_scores=prefill_scores, evict_to_other_blocks=evict_to_other_blocks,
                evict_in_place=evict_in_place)


NAMES = ["window_decode", "window_prefill", "decode_scores", "prefill_scores", "evict_to_other_blocks", "evict_in_place"]


def same(a, b):
    """Bit for bit (NaN scores of poisoned slots included)."""
    return all(torch.equal(x.view(torch.int16) if x.dtype == torch.bfloat16 else x.view(torch.int32),
                           y.view(torch.int16) if y.dtype == torch.bfloat16 else y.view(torch.int32))
               for x, y in zip(a, b))


@pytest.mark.parametrize("name", NAMES)
def test_captured_and_replayed(name):
    """A captured call replayed several times, with eager calls between: every replay gives what
    the eager calls give after as many passes (scores add up, a second eviction chooses anew)."""
    make = calls()[name]
    print(f"[case] {name} captured", flush=True)
    written, run = make()
    eager, run_eager = make()
    side = torch.cuda.Stream()
    start = [x.clone() for x in written]
    with torch.cuda.stream(side):
        run()                                   # what a first call loads is loaded
    torch.cuda.synchronize()
    for x, y in zip(written, start):
        x.copy_(y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    torch.cuda.synchronize()
    for _ in range(4):
        graph.replay()
        run_eager()
        torch.cuda.synchronize()
        assert same(written, eager)


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


def test_all_at_once():
    """Every operator twice, on streams of their own, with nothing between them."""
    made = calls()
    print("[case] all operators at once", flush=True)
    want = {}
    for name in NAMES:
        want[name], run = made[name]()
        run()
    torch.cuda.synchronize()
    got = []
    for name in NAMES * 2:
        stream = torch.cuda.Stream()
        got.append((name, *made[name](stream=stream)))
    torch.cuda.synchronize()
    for _, _, run in got:
        run()
    torch.cuda.synchronize()
    for name, written, _ in got:
        assert same(written, want[name]), name


def test_pools_past_two_to_the_31_elements():
    """The same blocks at the end of a pool of 2.3e9 elements: the same results, bit for bit."""
    from paper_2608_14624_amd import ops
    hkv, hq, far = 8, 32, 140000
    lens = [700, 1500]
    pg = Paged(63, lens, hkv, D, spare=80)
    n = pg.num_blocks
    q = to_gpu(bf16_bits(pg.rng, 2, hq, D))
    qp = to_gpu(bf16_bits(pg.rng, 150, hq, D))
    scores = pg.rng.random((n, hkv, 16)).astype(np.float32)
    dst = pg.tables.copy()
    dst[0, :20], dst[1, :20] = pg.free[:20], pg.free[20:40]
    print(f"[case] pools of {far * hkv * 16 * D} elements", flush=True)
    results = []
    for offset in (0, far - n):
        total = n + offset
        k, v = (torch.empty(total, hkv, 16, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        s = torch.empty(total, hkv, 16, device="cuda")
        k[offset:], v[offset:], s[offset:] = to_gpu(pg.k), to_gpu(pg.v), to_gpu(scores)
        t, d, ld = to_gpu(pg.tables + np.int32(offset)), to_gpu(dst + np.int32(offset)), to_gpu(pg.lens)
        out, outs, outp = torch.empty_like(q), torch.empty_like(q), torch.empty_like(qp)
        ops.cs_decode_window_attn(q, k, v, t, ld, out, max_seq_len=1500, window=400, sinks=4, scale=SCALE)
        ops.cs_prefill_window_attn(qp, k, v, t, i32(650, 1400), i32(0, 50, 150), outp, max_q_len=100, max_kv_len=1500,
                                   window=400, sinks=4, scale=SCALE)
        ops.cs_prefill_key_scores(qp, k, t, i32(650, 1400), i32(0, 50, 150), i32(0, 0), s, max_q_len=100,
                                  max_kv_len=1500, rows=70, scale=SCALE, decay=0.5)
        ops.cs_decode_attn_scores(q, k, v, t, ld, i32(0, 0), s, outs, max_seq_len=1500, max_scored_len=1500,
                                  scale=SCALE, decay=0.5)
        kept, new = torch.zeros(2, hkv, 300, dtype=torch.int32, device="cuda"), torch.zeros_like(ld)
        ops.cs_kv_evict(s, k, v, t, d, ld, i32(0, 0), kept, new, max_seq_len=1500, budget=300, trigger=300, recent=9)
        ops.cs_kv_evict(s, k, v, t, None, ld, i32(0, 0), kept, new, max_seq_len=1500, budget=300, trigger=300, recent=9)
        torch.cuda.synchronize()
        results.append([x.clone() for x in (out, outp, outs, kept, new, k[offset:], v[offset:], s[offset:])])
        del k, v, s
    assert same(*results)


def test_rising_logits():
    """Logits that rise by hundreds along the keys: the statistics' reference has to move, and the
    weights of all but the last keys vanish.  (An exponent of 400 carries 16 roundings of 2^-24 of
    itself from the matrix product, 4e-4, once in a weight and once in its normaliser.)"""
    from paper_2608_14624_amd import ops
    n, rows = 1000, 40
    pg = Paged(64, [n], HKV, D)
    k = bf16_bits_to_f64(pg.k).astype(np.float32)
    q = bf16_bits(pg.rng, rows, HQ, D)
    lift = np.zeros((D,), dtype=np.float32)
    lift[0] = 1.0
    for j in range(n):                     # every query's first feature is 16, the keys' rises to 280
        k[pg.tables[0, j // 16], :, j % 16, 0] = 280.0 * j / n
    bits = to_gpu(k).bfloat16()
    q = bf16_bits_to_f64(q)
    q[:, :, 0] = 16.0
    q = to_bits(to_gpu(q.astype(np.float32)).bfloat16())
    pg.k[:] = to_bits(bits)
    pg.k[pg.tables[0, n // 16], :, n % 16:] = 0x7FC0
    s = np.zeros((pg.num_blocks, HKV, 16), dtype=np.float32)
    print("[case] rising logits", flush=True)
    sd, so = to_gpu(s), to_gpu(s)
    ops.cs_prefill_key_scores(to_gpu(q), to_gpu(pg.k), to_gpu(pg.tables), i32(n - rows), i32(0, rows), i32(0), sd,
                              max_q_len=rows, max_kv_len=n, rows=rows, scale=SCALE)
    out = torch.empty(1, HQ, D, dtype=torch.bfloat16, device="cuda")
    ops.cs_decode_attn_scores(to_gpu(q[-1:]), to_gpu(pg.k), to_gpu(pg.v), to_gpu(pg.tables), i32(n), i32(0), so, out,
                              max_seq_len=n, max_scored_len=n, scale=SCALE)
    torch.cuda.synchronize()
    for got, first in ((sd, n - rows), (so, n - 1)):
        want = np.zeros(s.shape)
        add_key_scores(want, q[first - n:], pg.k, pg.tables[0], first, first, 0, HQ, HKV, SCALE, 1.0)
        err = np.abs(got.cpu().numpy() - want)
        assert (err <= 1e-3 * want + 1e-7).all(), err.max()


def test_outputs_of_any_alignment():
    """Decode outputs that are not 16-byte aligned."""
    from paper_2608_14624_amd import ops
    pg = Paged(65, [700, 40], HKV, D)
    q = bf16_bits(pg.rng, 2, HQ, D)
    out = torch.empty(2 * HQ * D + 1, dtype=torch.bfloat16, device="cuda")[1:].view(2, HQ, D)
    outs = torch.empty(2 * HQ * D + 1, dtype=torch.bfloat16, device="cuda")[1:].view(2, HQ, D)
    scores = np.zeros((pg.num_blocks, HKV, 16), dtype=np.float32)
    sd = to_gpu(scores)
    print("[case] outputs at odd addresses", flush=True)
    args = [to_gpu(q), to_gpu(pg.k), to_gpu(pg.v), to_gpu(pg.tables), to_gpu(pg.lens)]
    ops.cs_decode_window_attn(*args, out, max_seq_len=700, window=300, sinks=3, scale=SCALE)
    ops.cs_decode_attn_scores(*args, i32(0, 0), sd, outs, max_seq_len=700, max_scored_len=700, scale=SCALE)
    torch.cuda.synchronize()
    for r, n in enumerate([700, 40]):
        for x, kw in ((out, dict(window=300, sinks=3)), (outs, {})):
            ref, mag = window_attention(q[r:r + 1], pg.k, pg.v, pg.tables[r], n - 1, HQ, HKV, SCALE, **kw)
            assert (np.abs(bf16_bits_to_f64(to_bits(x[r:r + 1])) - ref) <= attention_bound(ref, mag)).all()
        want = scores.astype(np.float64)
        add_key_scores(want, q[r:r + 1], pg.k, pg.tables[r], n - 1, n - 1, 0, HQ, HKV, SCALE, 1.0)
        j = np.arange(n)
        at = pg.tables[r, j // 16], slice(None), j % 16
        assert (np.abs(sd.cpu().numpy()[at] - want[at]) <= weight_bound(want[at])).all()


@pytest.mark.parametrize("name", ["window_decode", "window_prefill", "decode_scores", "prefill_scores"])
def test_a_workspace_too_small_is_refused(name):
    from paper_2608_14624_amd import ops
    print(f"[case] {name} with too small a workspace", flush=True)
    written, run = calls()[name](workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    before = [x.clone() for x in written]
    with pytest.raises(ops.CacheScoutError, match="workspace_bytes"):
        run()
    _, run = calls()[name](workspace="automatic")
    with pytest.raises(ops.CacheScoutError, match="workspace"):
        run()
    torch.cuda.synchronize()
    assert same(written, before)


def test_debug_checks(monkeypatch):
    """With CS_DEBUG_CHECK=1 metadata that the calls forbid is refused before anything runs."""
    from paper_2608_14624_amd import ops
    monkeypatch.setenv("CS_DEBUG_CHECK", "1")
    pg = Paged(66, [200, 300], HKV, D, spare=30)
    kd, vd, ld = to_gpu(pg.k), to_gpu(pg.v), to_gpu(pg.lens)
    sd = to_gpu(np.zeros((pg.num_blocks, HKV, 16), dtype=np.float32))
    q = to_gpu(bf16_bits(pg.rng, 2, HQ, D))
    out = torch.empty_like(q)
    print("[case] debug checks", flush=True)

    def decode(tables=pg.tables, lens=ld, frm=i32(0, 0)):
        ops.cs_decode_attn_scores(q, kd, vd, to_gpu(tables), lens, frm, sd, out, max_seq_len=300, max_scored_len=300,
                                  scale=SCALE)

    def prompt(tables=pg.tables, frm=i32(0, 0)):
        ops.cs_prefill_key_scores(q, kd, to_gpu(tables), i32(199, 299), i32(0, 1, 2), frm, sd, max_q_len=1,
                                  max_kv_len=300, rows=3, scale=SCALE)

    def evicts(dst, tables=pg.tables, lens=ld):
        kept = torch.empty(2, HKV, 100, dtype=torch.int32, device="cuda")
        ops.cs_kv_evict(sd, kd, vd, to_gpu(tables), None if dst is None else to_gpu(dst), lens, i32(0, 16), kept,
                        torch.empty_like(ld), max_seq_len=300, budget=100, trigger=150, recent=4)

    def window(tables=pg.tables, lens=ld, **kw):
        ops.cs_decode_window_attn(q, kd, vd, to_gpu(tables), lens, out, max_seq_len=300, scale=SCALE,
                                  **{"window": 64, "sinks": 4, **kw})

    shared = pg.tables.copy()
    shared[1, 3] = shared[0, 3]
    outside = pg.tables.copy()
    outside[1, 6] = pg.num_blocks
    in_use, twice = pg.tables.copy(), pg.tables.copy()
    twice[0, :7], twice[1, 1:8] = pg.free[:7], pg.free[:7]
    for bad in (lambda: decode(tables=shared), lambda: decode(tables=outside), lambda: decode(lens=i32(200, 301)),
                lambda: decode(frm=i32(-1, 0)), lambda: prompt(tables=shared), lambda: prompt(frm=i32(0, -2)),
                lambda: evicts(in_use), lambda: evicts(twice), lambda: evicts(None, tables=shared),
                lambda: evicts(None, lens=i32(-1, 3)), lambda: window(lens=i32(0, 301)),
                lambda: window(tables=outside, window=300)):
        with pytest.raises(ops.CacheScoutError, match="CS_ERR_INVALID_ARG"):
            bad()
    good = pg.tables.copy()
    good[0, :7], good[1, 1:8] = pg.free[:7], pg.free[7:14]
    decode()
    decode(tables=shared, frm=i32(64, 64))             # shared before what is scored
    prompt()
    window(tables=outside)                             # out of sight
    window(lens=i32(0, 300))
    evicts(good)
    evicts(good, tables=shared)                        # old blocks are only read
    evicts(None)
    torch.cuda.synchronize()


def test_debug_checks_leave_invocations_without_rows_alone(monkeypatch):
    """An invocation without suffix rows changes no score, so its blocks may be another's."""
    from paper_2608_14624_amd import ops
    monkeypatch.setenv("CS_DEBUG_CHECK", "1")
    pg = Paged(67, [200, 300], HKV, D)
    tables = np.concatenate([pg.tables[1:], pg.tables[1:], pg.tables[:1]])
    sd = to_gpu(np.zeros((pg.num_blocks, HKV, 16), dtype=np.float32))
    q = bf16_bits(pg.rng, 3, HQ, D)
    print("[case] debug checks of prompt scores with an invocation without rows", flush=True)
    run = lambda cu: ops.cs_prefill_key_scores(to_gpu(q), to_gpu(pg.k), to_gpu(tables), i32(298, 298, 199),
                                               i32(*cu), i32(0, 0, 0), sd, max_q_len=2, max_kv_len=300, rows=3,
                                               scale=SCALE)
    run([0, 0, 2, 3])
    run([0, 2, 2, 3])
    with pytest.raises(ops.CacheScoutError, match="CS_ERR_INVALID_ARG"):
        run([0, 1, 2, 3])
    torch.cuda.synchronize()
    want = np.zeros((pg.num_blocks, HKV, 16))
    for _ in range(2):
        add_key_scores(want, q[:2], pg.k, tables[0], 298, 298, 0, HQ, HKV, SCALE, 1.0)
        add_key_scores(want, q[2:], pg.k, tables[2], 199, 199, 0, HQ, HKV, SCALE, 1.0)
    check_scores(sd, want, tables[[0, 2]], [300, 200], 0)
