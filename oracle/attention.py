"""Causal attention of packed prompts, of chunks against the paged FP8 cache, and of decode batches that
share prefixes, in fp64 -- oracle, test infrastructure only.

Besides the result each function gives what a bound of a kernel's error takes: `mean_abs`, the values'
magnitudes weighted like the values, and `score`, the largest sum of magnitudes that any score adds up.
"""
import numpy as np

from . import e4m3, kv
from .quant import bf16_bits_to_f32


def _attend(q, k, v, limit, sm_scale):
    """q [heads][dim] at one position, k, v [n][kv][dim]; keys 0 .. limit: (out, mean_abs, score, largest value)."""
    heads, dim = q.shape
    out, mean_abs, score, big = np.zeros((heads, dim)), np.zeros((heads, dim)), np.zeros(heads), np.zeros(heads)
    if limit < 0:
        return out, mean_abs, score, big
    group = heads // k.shape[1]
    for h in range(heads):
        kh, vh = k[:limit + 1, h // group], v[:limit + 1, h // group]
        s = kh @ q[h] * sm_scale
        p = np.exp(s - s.max())
        p /= p.sum()
        out[h], mean_abs[h] = p @ vh, p @ np.abs(vh)
        score[h] = (np.abs(kh) @ np.abs(q[h])).max() * sm_scale
        big[h] = np.abs(vh).max()
    return out, mean_abs, score, big


def _rows(jobs, total, heads, dim):
    res = [np.full((total, heads, dim), np.nan), np.full((total, heads, dim), np.nan), np.full((total, heads), np.nan),
           np.full((total, heads), np.nan)]
    for row, args in jobs:
        for r, x in zip(res, _attend(*args)):
            r[row] = x
    return res


def prompt(q_bits, k_bits, v_bits, cu_seqlens, sm_scale):
    """[T][heads][dim] bf16 bits -> (out, mean_abs, score, big); NaN in rows of no sequence."""
    q, k, v = (bf16_bits_to_f32(np.asarray(x, np.uint16)).astype(np.float64) for x in (q_bits, k_bits, v_bits))
    jobs = [(int(a) + i, (q[a + i], k[a:b], v[a:b], i, sm_scale)) for a, b in zip(cu_seqlens[:-1], cu_seqlens[1:])
            for i in range(int(b) - int(a))]
    return _rows(jobs, *q.shape)


def prompt_paged(q_bits, k_cache, v_cache, k_scale, v_scale, block_table, seq_lens, cu_seqlens, sm_scale):
    """The last cu[b + 1] - cu[b] of each sequence's seq_lens[b] cached tokens."""
    q = bf16_bits_to_f32(np.asarray(q_bits, np.uint16)).astype(np.float64)
    jobs = []
    for b, n in enumerate(int(x) for x in seq_lens):
        k = e4m3.decode(kv.gather_sequence(k_cache, block_table[b], n)).astype(np.float64) * float(k_scale)
        v = e4m3.decode(kv.gather_sequence(v_cache, block_table[b], n)).astype(np.float64) * float(v_scale)
        new = int(cu_seqlens[b + 1]) - int(cu_seqlens[b])
        jobs += [(int(cu_seqlens[b]) + i, (q[cu_seqlens[b] + i], k, v, n - new + i, sm_scale)) for i in range(new)]
    return _rows(jobs, *q.shape)


def shared_table(block_table, seq_lens, group_offsets, prefix_lens, max_prefix_len):
    """The block table as the sequences of a group see it: the shared blocks by the group's first row."""
    table = np.array(block_table)
    for g in range(len(prefix_lens)):
        a, b = int(group_offsets[g]), int(group_offsets[g + 1])
        if a < b:
            pages = max(0, min(int(prefix_lens[g]), max_prefix_len, int(seq_lens[a]))) // kv.BLOCK_TOKENS
            table[a:b, :pages] = table[a, :pages]
    return table


def bound(res, keys, half_step, floor):
    """How far a kernel's output may be from `res` = (out, mean_abs, score, big).

    With p_t = e^(s_t - m) and sums over at most `keys` terms, in fp32 (u = 2^-24):
      * a score is off by at most 130 u score (128 products and sums, the factor), its exponent by as much again
        for the rounded factor and maximum, and e^x by 4 u: every p_t by d = u (260 score + 8), relative;
      * P in the value product is rounded by half_step, relative, or by half of `floor` where that is more (fp16's
        smallest step, 2^-24, over the 2^7 by which weights are multiplied there; p = 1 at the maximum, so the sum is at
        least 1): half_step mean_abs + keys floor/2 big;
      * the sums of p v and of p add `keys` terms in fp32, in products of 16 and by rescaling, each off by at most
        keys u: 2 keys u mean_abs, and d counts for both: 2 d mean_abs; joining records adds 16 u;
      * the output is rounded once to bf16: 2^-8 |out|, on top of the rest.
    """
    out, mean_abs, score, big = res
    u = 2.0 ** -24
    d = u * (260.0 * score[..., None] + 8.0)
    before = mean_abs * (half_step + 2.0 * d + 2.0 * keys * u + 16.0 * u) + 0.5 * keys * floor * big[..., None]
    return before + 2.0 ** -8 * (np.abs(out) + before) + 2.0 ** -133


BF16_VALUES = (2.0 ** -8, 0.0)                # half_step, floor of P against bf16 values (bf16 underflows like fp32)
FP8_VALUES = (2.0 ** -11, 2.0 ** -31)         # of 2^7 P in fp16 against codes
