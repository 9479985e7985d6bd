"""Blocks entered and counted ahead of their tokens: free and compact take lengths that cover them, attention and fork the
sequences' own."""
import numpy as np
import pytest
import torch

from oracle import attention, pages
from tests.attn_util import bf16, check, codes, f32_1, i32
from tests.gpu_util import announce, need_gpu, u16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fp8rl():
    need_gpu()
    import paper_2601_18150_amd as m
    m.load()
    return m


def ahead(rng, lens, kv_heads, width, blocks):
    """Caches of random codes, a table in which every row has room for its next token, and the lengths that cover it."""
    held = [(n // 16 + 1) * 16 if n % 16 == 0 else n for n in lens]
    table = rng.integers(-3, blocks + 3, (len(lens), width)).astype(np.int32)
    free, refs = list(rng.permutation(blocks)), np.zeros(blocks, np.int32)
    for r, n in enumerate(held):
        used = (n + 15) // 16
        table[r, :used], free = free[:used], free[used:]
        refs[table[r, :used]] = 1
    kc, vc = codes(rng, (blocks, kv_heads, 16, 128)), codes(rng, (blocks, kv_heads, 4, 128, 4))
    return kc, vc, table, np.array(lens, np.int32), np.array(held, np.int32), refs


def test_next_tokens_after_free_and_compact(fp8rl):
    announce("free and compact with blocks ahead, the next token of every sequence, a fork of one")
    rng = np.random.default_rng(1)
    kv_heads, heads, blocks, sm = 2, 8, 40, 0.09
    kc, vc, table, lens, held, refs = ahead(rng, [32, 48, 20, 16, 96, 0], kv_heads, 8, blocks)
    before = [[c[table[r, :(held[r] + 15) // 16]].copy() for c in (kc, vc)] for r in range(6)]
    gkc, gvc = torch.from_numpy(kc.copy()).cuda(), torch.from_numpy(vc.copy()).cuda()
    t, ln, hd, rf = (torch.from_numpy(x.copy()).cuda() for x in (table, lens, held, refs))
    fp8rl.fp8rl_kv_free_sequences(t, hd, rf, i32([1, 3]))
    ln[[1, 3]] = 0
    live = fp8rl.fp8rl_kv_compact([gkc, gvc], t, hd, rf)
    torch.cuda.synchronize()
    pages.free(table, held, refs, [1, 3])
    want = pages.compact([kc, vc], table, held, refs)
    assert int(live) == want == 3 + 2 + 7 + 1 and np.array_equal(hd.cpu().numpy(), held)
    assert np.array_equal(t.cpu().numpy(), table) and np.array_equal(rf.cpu().numpy(), refs)
    assert np.array_equal(gkc.cpu().numpy(), kc) and np.array_equal(gvc.cpu().numpy(), vc)
    left = [0, 2, 4, 5]
    for r in left:                                         # every block of a row, the one ahead too, is where the table says
        named = table[r, :(held[r] + 15) // 16]
        assert np.all(named < want) and np.all(refs[named] == 1)
        assert np.array_equal(kc[named], before[r][0]) and np.array_equal(vc[named], before[r][1])

    rows, one = torch.tensor(left, device="cuda"), f32_1(1.0)
    at = ln[rows].long()
    slot = t[rows].gather(1, (at // 16)[:, None])[:, 0].long() * 16 + at % 16
    q, k, v = bf16(rng, (4, heads, 128)), bf16(rng, (4, kv_heads, 128)), bf16(rng, (4, kv_heads, 128))
    fp8rl.fp8rl_kv_cache_write_fp8(k.cuda(), v.cuda(), slot, one, one, gkc, gvc)
    ln[rows] += 1
    out = fp8rl.fp8rl_attention_prompt_fp8kv(q.cuda(), gkc, gvc, t[rows].contiguous(), ln[rows].contiguous(), i32(range(5)), 128,
                                             one, one, sm)
    torch.cuda.synchronize()
    now = [lens[r] + 1 for r in left]
    res = attention.prompt_paged(u16(q), gkc.cpu().numpy(), gvc.cpu().numpy(), 1.0, 1.0, table[left], now, np.arange(5), sm)
    check(out, res, 97, attention.FP8_VALUES, "the next tokens")

    fp8rl.fp8rl_kv_fork_sequences([gkc, gvc], t, ln, rf, i32([0]), i32([1]), i32([want]))
    torch.cuda.synchronize()
    child = t[1].cpu().numpy()
    assert int(ln[1]) == 33 and list(child[:3]) == [table[0, 0], table[0, 1], want]
    assert torch.equal(gkc[want], gkc[int(table[0, 2])]) and int(rf[want]) == 1 and int(rf[int(table[0, 0])]) == 2


def test_lengths_that_do_not_cover_a_block():
    """(Why: the same by the oracle, with the sequences' own lengths, leaves the block ahead where the table does not say.)"""
    rng = np.random.default_rng(2)
    kc, vc, table, lens, held, refs = ahead(rng, [32, 16], 1, 4, 20)
    assert pages.compact([kc, vc], table, lens, refs) == 5
    assert table[0, 2] >= 5 or table[1, 1] >= 5            # a block that is free now
