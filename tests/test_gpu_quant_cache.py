"""The write-back into a pool held in 4 or 8 bits, and whole blocks into such a pool and back,
against the oracle: codes and scales exactly, for every bf16 number, and nothing else touched."""

import numpy as np
import pytest

from bounded_cache_util import bf16_bits, to_bits, to_gpu
from oracle import bf16_bits_to_f64, pack_tiles, quantise_rows, row_values, split_tiles, to_bf16_bits, unpack_tiles
from quant_util import spread_rows

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

FORMATS = [(64, 4), (64, 8), (128, 4), (128, 8)]
FILL = 0xA5


def i32(x):
    return to_gpu(np.asarray(x, dtype=np.int32))


def check_rows(tiles, at, k, v, d, bits):
    """Rows (block, head, offset) `at` of tiles hold k and v, code by code; a row's group that is not
    finite reads as NaN."""
    kc, ks, vc, vs = (x[at] for x in split_tiles(tiles, d, bits))
    for name, got_c, got_s, want in (("K", kc, ks, k), ("V", vc, vs, v)):
        codes, scales = quantise_rows(want, bits)
        assert (got_s == scales).all(), f"{name}: scales differ in {(got_s != scales).sum()} places"
        fine = (scales != 255).repeat(32, -1)
        assert (got_c[fine] == codes[fine]).all(), f"{name}: {(got_c != codes)[fine].sum()} codes differ"


@pytest.mark.parametrize("d,bits", FORMATS)
def test_every_bf16_number(d, bits):
    """In groups of its own power of two, and next to numbers of others; blocks into the pool and
    what they are read back as."""
    from paper_2608_14624_amd import ops
    print(f"[case] every number, head_dim {d}, {bits} bits", flush=True)
    rng = np.random.default_rng(1)
    every = np.arange(65536, dtype=np.uint32).astype(np.uint16)
    rows = np.concatenate([every, rng.permutation(every), np.sort(rng.permutation(every)[:32768])])
    blocks = rows.reshape(-1, 2, 16, d)
    n = blocks.shape[0]
    k, v = blocks, np.ascontiguousarray(blocks[::-1])
    pool = torch.full((n, 2, ops.kv_quant_tile_bytes(d, bits)), FILL, dtype=torch.uint8, device="cuda")
    kd, vd = to_gpu(k), to_gpu(v)
    order = rng.permutation(n)
    ops.cs_kv_quantize(kd, vd, i32(np.arange(n)), i32(order), pool, bits=bits)
    torch.cuda.synchronize()
    tiles = pool.cpu().numpy()
    b, h, t = np.meshgrid(order, np.arange(2), np.arange(16), indexing="ij")
    check_rows(tiles, (b, h, t), k, v, d, bits)
    back = torch.zeros(2, n, 2, 16, d, dtype=torch.bfloat16, device="cuda")
    ops.cs_kv_dequantize(pool, i32(order), i32(np.arange(n)), back[0], back[1], bits=bits)
    torch.cuda.synchronize()
    for got, x in zip(back, (k, v)):
        want = row_values(*quantise_rows(x, bits), bits)
        got = bf16_bits_to_f64(to_bits(got))
        same = (got == want) | (np.isnan(got) & np.isnan(want))
        assert same.all(), f"{(~same).sum()} values differ, first {x[~same][:4]} {got[~same][:4]} {want[~same][:4]}"


@pytest.mark.parametrize("d,bits", FORMATS)
@pytest.mark.parametrize("hkv,tokens", [(1, 1), (8, 1), (2, 15), (3, 16), (1, 17), (5, 100), (8, 333)])
def test_write_scatters_tokens(d, bits, hkv, tokens):
    """Slots in any order, some negative, starting inside blocks; every other byte stays."""
    from paper_2608_14624_amd import ops
    print(f"[case] write {tokens} tokens, {hkv} heads of {d}, {bits} bits", flush=True)
    rng = np.random.default_rng(tokens)
    blocks = tokens // 16 + 4
    k, v = spread_rows(rng, tokens, hkv, d), spread_rows(rng, tokens, hkv, d)
    if tokens > 20:      # runs of a sequence, from inside a block, and scattered tokens
        run = 5 + np.arange(tokens // 2)
        rest = rng.permutation(np.setdiff1d(np.arange(blocks * 16), run))[:tokens - len(run)]
        slots = np.concatenate([run, rest])
    else:
        slots = rng.permutation(blocks * 16)[:tokens]
    slots = np.where(rng.random(tokens) < 0.1, -1 - np.arange(tokens), slots) if tokens > 1 else slots
    size = ops.kv_quant_tile_bytes(d, bits)
    pool = torch.full((blocks, hkv, size), FILL, dtype=torch.uint8, device="cuda")
    ops.cs_kv_write_quant(to_gpu(k), to_gpu(v), i32(slots), pool, bits=bits)
    torch.cuda.synchronize()
    want = np.full((blocks, hkv, size), FILL, dtype=np.uint8)
    # the written rows, placed by the layout: packed alone, and taken over byte by byte.  A byte
    # belongs to one token alone, which the second packing shows
    live = slots >= 0
    full_k, full_v = np.zeros((2, blocks, hkv, 16, d), dtype=np.uint16)
    full_k[slots[live] // 16, :, slots[live] % 16] = k[live]
    full_v[slots[live] // 16, :, slots[live] % 16] = v[live]
    packed = pack_tiles(full_k, full_v, bits)
    other_k, other_v = (np.full_like(x, 0xBFC0) for x in (full_k, full_v))      # -1.5: no byte as of 0
    other_k[slots[live] // 16, :, slots[live] % 16] = 0
    other_v[slots[live] // 16, :, slots[live] % 16] = 0
    others = pack_tiles(other_k, other_v, bits) != pack_tiles(0 * other_k, 0 * other_v, bits)
    want = np.where(others, want, packed)
    got = pool.cpu().numpy()
    assert (got == want).all(), f"{(got != want).sum()} bytes differ"


@pytest.mark.parametrize("d,bits", FORMATS)
def test_repeats_order_and_bystanders(d, bits):
    """A source block that is named twice, places in any order, and what is not named left alone;
    the way back gives the same values twice."""
    from paper_2608_14624_amd import ops
    print(f"[case] blocks, head_dim {d}, {bits} bits", flush=True)
    rng = np.random.default_rng(7)
    k, v = bf16_bits(rng, 9, 3, 16, d), bf16_bits(rng, 9, 3, 16, d)
    size = ops.kv_quant_tile_bytes(d, bits)
    pool = torch.full((12, 3, size), FILL, dtype=torch.uint8, device="cuda")
    src, dst = [4, 0, 4, 8, 2], [11, 3, 0, 7, 5]
    ops.cs_kv_quantize(to_gpu(k), to_gpu(v), i32(src), i32(dst), pool, bits=bits)
    torch.cuda.synchronize()
    want = np.full((12, 3, size), FILL, dtype=np.uint8)
    want[dst] = pack_tiles(k[src], v[src], bits)
    assert (pool.cpu().numpy() == want).all()
    out = to_gpu(np.stack([k, v]))
    ops.cs_kv_dequantize(pool, i32([11, 11, 7]), i32([1, 6, 2]), out[0], out[1], bits=bits)
    torch.cuda.synchronize()
    for got, x in zip(out, (k, v)):
        ref = x.copy()
        ref[[1, 6, 2]] = to_bf16_bits(row_values(*quantise_rows(x[[4, 4, 8]], bits), bits))
        assert (bf16_bits_to_f64(to_bits(got)) == bf16_bits_to_f64(ref)).all()


@pytest.mark.parametrize("d,bits", FORMATS)
def test_any_bytes_are_read(d, bits):
    """Tiles of random bytes with scales from the smallest written to the largest, and NaN: the way
    back gives what they stand for."""
    from paper_2608_14624_amd import ops
    print(f"[case] any bytes, head_dim {d}, {bits} bits", flush=True)
    rng = np.random.default_rng(9)
    n = 40
    tiles = rng.integers(0, 256, (n, 2, ops.kv_quant_tile_bytes(d, bits)), dtype=np.uint8)
    lo, hi = {4: (2, 252), 8: (10, 246)}[bits]
    at = 4 * d * bits
    tiles[:, :, at:] = np.where(rng.random((n, 2, d)) < 0.05, 255, rng.integers(lo, hi + 1, (n, 2, d)))
    out = torch.zeros(2, n, 2, 16, d, dtype=torch.bfloat16, device="cuda")
    ids = rng.permutation(n)
    ops.cs_kv_dequantize(to_gpu(tiles), i32(ids), i32(np.arange(n)), out[0], out[1], bits=bits)
    torch.cuda.synchronize()
    for got, want in zip(out, unpack_tiles(tiles[ids], d, bits)):
        got = bf16_bits_to_f64(to_bits(got))
        assert ((got == want) | (np.isnan(got) & np.isnan(want))).all()
