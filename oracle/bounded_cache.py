"""Float64 oracles of the operators that bound a sequence's cache (test infrastructure).

Attention with a sliding window and sinks, the attention weights that keys
receive, and eviction by them.  Row ``i`` of an invocation is prompt position
``p = P + i``; under a window of ``window`` keys with ``sinks`` first tokens it sees
key ``j <= p`` if ``j > p - window`` or ``j < sinks``.  Pools, block tables and lengths
are those of ``paged_attention``.
"""

import numpy as np

from .paged_attention import bf16_bits_to_f64


def _rows(pool_bits, slots, offsets, g):
    return bf16_bits_to_f64(pool_bits[slots, g, offsets])


def window_weights(q, k_pool, table, first_pos, num_rows, g, group, scale, window=None, sinks=0):
    """Softmax weights ``[group, rows, keys]`` of the rows at positions
    ``first_pos ..`` (``q``: their float64 queries of KV head g, ``[rows, group,
    D]``) over the keys they may see; only visible keys' blocks are looked up."""
    n = first_pos + num_rows
    bs = k_pool.shape[2]
    keys = np.arange(n)
    pos = first_pos + np.arange(num_rows)[:, None]
    see = keys[None, :] <= pos
    if window is not None:
        see &= (keys[None, :] > pos - window) | (keys[None, :] < sinks)
    used = np.flatnonzero(see.any(0))
    k = _rows(k_pool, np.asarray(table)[used // bs], used % bs, g)
    logits = np.full((group, num_rows, n), -np.inf)
    logits[:, :, used] = np.einsum("rhd,kd->hrk", q, k) * float(np.float32(scale))
    logits[:, ~see] = -np.inf
    w = np.exp(logits - logits.max(-1, keepdims=True))
    return w / w.sum(-1, keepdims=True), used


def window_attention(q_bits, k_pool, v_pool, table, first_pos, hq, hkv, scale, window=None, sinks=0,
                     heads=None):
    """Output of one invocation's rows ``[rows, heads, D]`` and, for error
    bounds, the same with the absolute values of V."""
    group = hq // hkv
    bs = k_pool.shape[2]
    num_rows = q_bits.shape[0]
    heads = list(range(hq)) if heads is None else list(heads)
    out = np.zeros((num_rows, len(heads), q_bits.shape[2]))
    mag = np.zeros_like(out)
    for x, h in enumerate(heads):
        g = h // group
        w, used = window_weights(bf16_bits_to_f64(q_bits[:, h:h + 1]), k_pool, table, first_pos, num_rows, g, 1,
                                 scale, window, sinks)
        v = _rows(v_pool, np.asarray(table)[used // bs], used % bs, g)
        out[:, x] = w[0][:, used] @ v
        mag[:, x] = w[0][:, used] @ np.abs(v)
    return out, mag


def add_key_scores(scores, q_bits, k_pool, table, first_pos, new_from, score_from, hq, hkv, scale, decay):
    """Add the weights of the rows at positions ``first_pos ..`` to one
    sequence's scores (float64 ``[num_blocks, Hkv, block_size]``, in place): keys
    from ``new_from`` on start anew, keys before ``score_from`` are not scored."""
    group = hq // hkv
    bs = k_pool.shape[2]
    num_rows = q_bits.shape[0]
    n = first_pos + num_rows
    for g in range(hkv):
        w, _ = window_weights(bf16_bits_to_f64(q_bits[:, g * group:(g + 1) * group]), k_pool, table, first_pos,
                              num_rows, g, group, scale)
        total = w.sum((0, 1))
        for j in range(score_from, n):
            at = (table[j // bs], g, j % bs)
            scores[at] = total[j] + (decay * scores[at] if j < new_from else 0.0)


def evict(scores, k_pool, v_pool, table, dst_table, length, keep_from, budget, trigger, recent):
    """Evict from one sequence (pools and scores in place); the kept keys per KV
    head, or None where nothing is evicted, and the new length."""
    if length - keep_from <= trigger:
        return None, length
    bs = k_pool.shape[2]
    moving = dst_table is not None
    target = table if dst_table is None else dst_table
    kept = []
    for g in range(k_pool.shape[1]):
        competing = range(keep_from, length - recent)
        order = sorted(competing, key=lambda j: (_last_if_nan(scores[table[j // bs], g, j % bs]), j))
        keep = sorted(order[:budget - recent]) + list(range(length - recent, length))
        kept.append(keep)
        src = list(range(keep_from // bs * bs, keep_from)) + keep if moving else keep
        dst = range(keep_from // bs * bs if moving else keep_from, keep_from + budget)
        for pool in (k_pool, v_pool, scores):
            rows = [pool[table[j // bs], g, j % bs].copy() for j in src]
            for j, row in zip(dst, rows):
                pool[target[j // bs], g, j % bs] = row
    return np.array(kept, dtype=np.int32), keep_from + budget


def _last_if_nan(score):
    return np.inf if np.isnan(score) else -score
