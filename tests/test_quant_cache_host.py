"""Refusals and workspace sizes of the calls on a pool held in 4 or 8 bits, on the CPU: every call
here returns from its argument checks, or is a documented no-op, before any GPU work."""

import pytest

ops = pytest.importorskip("paper_2608_14624_amd.ops",
                          reason="libcachescout.so not built (run __graft_entry__.build())")

FAKE = 1 << 20   # a 16-byte aligned non-null address; never dereferenced here
BAD, UNSUPPORTED = ops.CS_ERR_INVALID_ARG, ops.CS_ERR_UNSUPPORTED

POOL = dict(num_kv_heads=2, head_dim=64, block_size=16, bits=4)
WRITE = dict(k_new=FAKE, v_new=FAKE, slot_mapping=FAKE, num_tokens=5, quant_pool=FAKE, num_blocks=8, **POOL)
BLOCKS = dict(k_pool=FAKE, v_pool=FAKE, src_block_ids=FAKE, dst_block_ids=FAKE, n=3, quant_pool=FAKE, num_blocks=8,
              num_quant_blocks=6, **POOL)
DECODE = dict(q=FAKE, quant_pool=FAKE, block_tables=FAKE, seq_lens=FAKE, batch=3, max_seq_len=48,
              max_blocks_per_seq=3, num_blocks=64, num_q_heads=8, **POOL, scale=0.125, workspace=FAKE,
              workspace_bytes=0, out=FAKE)
PREFILL = dict(q=FAKE, quant_pool=FAKE, block_tables=FAKE, prefix_lens=FAKE, cu_q_lens=FAKE, batch=2, total_q=10,
               max_q_len=8, max_kv_len=40, max_blocks_per_seq=3, num_blocks=64, num_q_heads=8, **POOL, scale=0.125,
               workspace=None, workspace_bytes=0, out=FAKE)
CALLS = {
    "write": (ops.cs_kv_write_quant_raw, WRITE),
    "quantize": (ops.cs_kv_quantize_raw, BLOCKS),
    "dequantize": (ops.cs_kv_dequantize_raw, BLOCKS),
    "decode": (ops.cs_decode_quant_attn_raw, DECODE),
    "prefill": (ops.cs_prefill_quant_attn_raw, PREFILL),
}


def call(name, **kw):
    fn, good = CALLS[name]
    assert set(kw) <= set(good)
    return fn(**dict(good, **kw))


COMMON = [(dict(num_blocks=-1), BAD), (dict(num_blocks=0), BAD), (dict(num_kv_heads=0), BAD),
          (dict(head_dim=96), UNSUPPORTED), (dict(head_dim=0), BAD), (dict(block_size=32), UNSUPPORTED),
          (dict(bits=2), UNSUPPORTED), (dict(bits=0), UNSUPPORTED), (dict(bits=16), UNSUPPORTED),
          (dict(quant_pool=None), BAD), (dict(quant_pool=FAKE + 8), BAD)]
COPY = [(dict(n=-1), BAD), (dict(num_quant_blocks=-1), BAD), (dict(num_quant_blocks=0), BAD),
        (dict(src_block_ids=None), BAD), (dict(dst_block_ids=None), BAD), (dict(k_pool=None), BAD),
        (dict(v_pool=None), BAD), (dict(k_pool=FAKE + 8), BAD), (dict(v_pool=FAKE + 2), BAD),
        # 2^32 threads
        (dict(n=2 ** 23, num_blocks=2 ** 23, num_quant_blocks=2 ** 23, num_kv_heads=4), BAD)]
ATTENTION = [(dict(batch=-1), BAD), (dict(max_blocks_per_seq=-1), BAD), (dict(max_blocks_per_seq=2), BAD),
             (dict(num_kv_heads=3), BAD), (dict(num_q_heads=0), BAD), (dict(scale=float("nan")), BAD),
             (dict(scale=float("inf")), BAD), (dict(scale=0.0), UNSUPPORTED), (dict(scale=-0.5), UNSUPPORTED),
             (dict(q=None), BAD), (dict(q=FAKE + 2), BAD), (dict(block_tables=None), BAD), (dict(out=None), BAD),
             (dict(out=FAKE + 8), BAD), (dict(workspace_bytes=-1), BAD)]
REFUSALS = {
    "write": COMMON + [(dict(num_tokens=-1), BAD), (dict(k_new=None), BAD), (dict(v_new=None), BAD),
                       (dict(slot_mapping=None), BAD), (dict(k_new=FAKE + 8), BAD), (dict(v_new=FAKE + 4), BAD),
                       (dict(num_tokens=2 ** 31 - 1, num_kv_heads=2), BAD)],
    "quantize": COMMON + COPY + [(dict(n=7), BAD)],
    "dequantize": COMMON + COPY + [(dict(n=9), BAD)],
    "decode": COMMON + ATTENTION + [(dict(num_q_heads=34), UNSUPPORTED), (dict(max_seq_len=-1), BAD),
                                    (dict(max_seq_len=0), BAD), (dict(seq_lens=None), BAD),
                                    (dict(batch=2 ** 24), BAD)],
    "prefill": COMMON + ATTENTION + [(dict(total_q=-1), BAD), (dict(max_q_len=-1), BAD), (dict(max_q_len=41), BAD),
                                     (dict(max_kv_len=-1), BAD), (dict(prefix_lens=None), BAD),
                                     (dict(cu_q_lens=None), BAD)],
}


@pytest.mark.parametrize("name,kw,status", [(n, kw, st) for n, cases in REFUSALS.items() for kw, st in cases])
def test_bad_arguments_are_refused(name, kw, status):
    assert call(name, **kw) == status
    assert ops.last_error() != ""


@pytest.mark.parametrize("name,kw", [
    ("write", dict(num_tokens=0)), ("write", dict(num_tokens=0, k_new=None, num_blocks=0)),
    ("quantize", dict(n=0)), ("quantize", dict(n=0, k_pool=None, quant_pool=None)), ("dequantize", dict(n=0)),
    ("decode", dict(batch=0)), ("decode", dict(batch=0, q=None, out=None)), ("prefill", dict(batch=0)),
    ("prefill", dict(total_q=0)), ("prefill", dict(max_q_len=0, q=None))])
def test_empty_work_is_a_noop(name, kw):
    assert call(name, **kw) == ops.CS_OK
    assert ops.last_error() == ""


def test_tile_bytes():
    assert [ops.kv_quant_tile_bytes(d, b) for d in (64, 128) for b in (4, 8)] == [1088, 2112, 2176, 4224]
    for d, b in [(96, 4), (128, 2), (0, 4), (128, 16), (-64, 8)]:
        assert ops.kv_quant_tile_bytes(d, b) == -1


def test_workspace_sizes():
    assert ops.decode_quant_workspace_bytes(3, 6000, 32, 8, 128, 256) > 0
    assert ops.decode_quant_workspace_bytes(0, 6000, 32, 8, 128, 256) == 0
    assert ops.prefill_quant_workspace_bytes(0, 0, 0, 0, 32, 8, 128, 256) == 0
    # a launch that fills the device needs none, a short suffix on a long prefix does
    assert ops.prefill_quant_workspace_bytes(16, 16 * 512, 512, 4608, 64, 8, 128, 256) == 0
    assert ops.prefill_quant_workspace_bytes(1, 8, 8, 4608, 32, 8, 128, 256) > 0
    for bad in (dict(batch=-1), dict(num_q_heads=9), dict(head_dim=96), dict(num_kv_heads=0), dict(num_cus=-1)):
        good = dict(batch=3, max_seq_len=6000, num_q_heads=32, num_kv_heads=8, head_dim=128, num_cus=256)
        assert ops.decode_quant_workspace_bytes(**{**good, **bad}) == -1
        good = dict(batch=3, total_q=9, max_q_len=5, max_kv_len=6000, num_q_heads=32, num_kv_heads=8, head_dim=128,
                    num_cus=256)
        assert ops.prefill_quant_workspace_bytes(**{**good, **bad}) == -1
    # lengths whose units of 64 sequences, or launches whose threads, would not fit 32 bits
    assert ops.decode_quant_workspace_bytes(1, 2 ** 30, 32, 8, 128, 256) == -1
    assert ops.decode_quant_workspace_bytes(2 ** 24, 100, 32, 8, 128, 256) == -1
    assert ops.prefill_quant_workspace_bytes(2 ** 16, 2 ** 30, 2 ** 14, 2 ** 14, 32, 8, 128, 256) == -1
    assert ops.prefill_quant_workspace_bytes(1, 8, 8, 0x7fffff00, 32, 8, 128, 256) == -1
    assert ops.prefill_quant_workspace_bytes(1, 8, 8, 0x7ffffeff, 32, 8, 128, 256) > 0
