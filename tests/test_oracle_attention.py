"""The fp64 oracle of prompt, chunk and shared-prefix attention against torch's attention in fp64, and the page oracle
by what it has to keep: every sequence's contents."""
import numpy as np
import pytest
import torch

from oracle import attention, e4m3, kv, pages
from oracle.quant import bf16_bits_to_f32
from tests.attn_util import bf16, codes, offsets, paged
from tests.gpu_util import u16


@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (8, 2), (8, 1)])
def test_prompt_is_torchs_causal_attention(heads, kv_heads):
    rng = np.random.default_rng(heads)
    lengths = [5, 0, 1, 33]
    cu = offsets(lengths, 2)
    q, k, v = (bf16(rng, (43, h, 128)) for h in (heads, kv_heads, kv_heads))
    out, mean_abs, score, _ = attention.prompt(u16(q), u16(k), u16(v), cu, 0.09)
    for a, b in zip(cu[:-1], cu[1:]):
        want = torch.nn.functional.scaled_dot_product_attention(
            *(x[a:b].double().transpose(0, 1)[None] for x in (q, k, v)), is_causal=True, scale=0.09, enable_gqa=True)
        assert np.allclose(out[a:b], want[0].transpose(0, 1).numpy(), rtol=1e-12, atol=1e-13)
    assert np.isnan(out[:2]).all() and np.isnan(out[41:]).all()
    assert np.all(mean_abs[2:41] >= np.abs(out[2:41]) - 1e-12) and np.all(score[2:41] > 0)


def test_paged_prompt_is_decode_of_every_token():
    rng = np.random.default_rng(1)
    lens, new = [40, 3, 17], [7, 5, 17]
    kc, vc, table = paged(rng, lens, 2)
    cu = offsets(new)
    q = u16(bf16(rng, (sum(new), 4, 128)))
    out = attention.prompt_paged(q, kc, vc, 0.5, 0.25, table, lens, cu, 0.01)[0]
    for b, n in enumerate(new):
        for i in range(n):
            at = lens[b] - n + i + 1
            want = kv.attention_decode(q[cu[b] + i][None], kc, vc, 0.5, 0.25, table[b][None], [max(at, 0)], 0.01)
            assert np.allclose(out[cu[b] + i], want[0], rtol=1e-12, atol=1e-12)


def test_bound_covers_a_rounded_softmax():
    """P rounded to bf16 stays inside the bound on the CPU too, and a key left out does not."""
    rng = np.random.default_rng(2)
    q, k, v = (bf16(rng, (50, 1, 128)) for _ in range(3))
    res = attention.prompt(u16(q), u16(k), u16(v), [0, 50], 0.09)
    s = (q[:, 0].float() @ k[:, 0].float().t() * 0.09).masked_fill(torch.ones(50, 50).triu(1) > 0, -torch.inf)
    p = torch.exp(s - s.amax(1, keepdim=True))
    near = ((p.bfloat16().float() @ v[:, 0].float()) / p.sum(1, keepdim=True)).bfloat16().double().numpy()
    limit = attention.bound(res, 50, *attention.BF16_VALUES)[:, 0]
    assert np.all(np.abs(near - res[0][:, 0]) <= limit)
    p[:, 3] = 0
    far = ((p @ v[:, 0].float()) / p.sum(1, keepdim=True)).double().numpy()
    assert (np.abs(far - res[0][:, 0]) > limit)[5:].any(1).all()


def contents(caches, table, lens, row):
    return [c[table[row, :(lens[row] + 15) // 16]] for c in caches]


def test_pages_keep_every_sequences_contents():
    rng = np.random.default_rng(3)
    caches = [codes(rng, (64, 2, 8)) for _ in range(3)]
    table, lens, refs = np.full((12, 6), -1, np.int32), np.zeros(12, np.int32), np.zeros(64, np.int32)
    blocks = list(rng.permutation(64))
    for r, n in enumerate((33, 16, 96)):
        used = (n + 15) // 16
        table[r, :used], lens[r] = blocks[:used], n
        refs[blocks[:used]] = 1
        blocks = blocks[used:]
    pages.fork(caches, table, lens, refs, [0, 0, 1, 2, 3, 0], [3, 4, 5, 6, 3, 40], blocks[:6])
    assert lens[3] == lens[4] == 33 and lens[5] == 16 and lens[6] == 96 and lens[7] == 0
    for parent, child in ((0, 3), (0, 4), (1, 5), (2, 6)):
        for a, b in zip(contents(caches, table, lens, parent), contents(caches, table, lens, child)):
            assert np.array_equal(a, b)
    assert table[3, 2] != table[0, 2] and refs[table[0, 0]] == 3 and refs[table[3, 2]] == 1
    assert (refs > 0).sum() == 3 + 1 + 6 + 2
    pages.free(table, lens, refs, [0, 2, 2, 99, -1])
    before = {r: contents(caches, table, lens, r) for r in range(12) if lens[r]}
    live = pages.compact(caches, table, lens, refs)
    assert live == (refs > 0).sum() and np.all(refs[:live] > 0) and np.all(refs[live:] == 0)
    for r, want in before.items():
        for a, b in zip(want, contents(caches, table, lens, r)):
            assert np.array_equal(a, b)
