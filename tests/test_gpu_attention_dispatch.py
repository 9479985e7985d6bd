"""The ways of attention's dispatch that need many rows: the 128-row bf16 tiles over many tiles of keys, more than 256
sequences or groups whose places are whole large tiles, and thousands of sequences (a third level of the search)."""
import numpy as np
import pytest
import torch

from oracle import attention
from tests.attn_util import bf16, check, f32_1, i32, offsets, paged
from tests.gpu_util import announce, need_gpu, u16

pytestmark = pytest.mark.gpu
KS, VS, SM = np.float32(0.02), np.float32(0.03), 0.02


@pytest.fixture(scope="module")
def fp8rl():
    need_gpu()
    import paper_2601_18150_amd as m
    m.load()
    return m


# more than 512 workgroups: 128 rows each
@pytest.mark.parametrize("heads,kv_heads,lengths", [(64, 64, [1100]), (64, 16, [1037, 77, 1]), (128, 64, [0, 333, 640, 128])])
def test_long_prompts_in_tiles_of_128_rows(fp8rl, heads, kv_heads, lengths):
    announce(f"prompt: {heads}/{kv_heads} heads, lengths {lengths}")
    rng = np.random.default_rng(heads + kv_heads)
    n, cu, group = sum(lengths), offsets(lengths), heads // kv_heads
    assert sum(-(-x * group // 128) for x in lengths) * kv_heads > 512
    # q, k and v as columns of one tensor, as a fused projection leaves them
    qkv = bf16(rng, (n, heads + 2 * kv_heads, 128))
    q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
    gpu = qkv.cuda()
    out = fp8rl.fp8rl_attention_prompt_bf16(gpu[:, :heads], gpu[:, heads:heads + kv_heads], gpu[:, heads + kv_heads:], i32(cu), 0.09)
    torch.cuda.synchronize()
    some = [0, kv_heads - 1]                               # (the oracle's time)
    mine = [h * group + g for h in some for g in (0, group - 1)]
    same = [h for h in some for _ in range(2)]
    res = attention.prompt(u16(q[:, mine]), u16(k[:, same]), u16(v[:, same]), cu, 0.09)
    check(out[:, mine], res, max(lengths), attention.BF16_VALUES, "prompt")


# runs of 86 rows and more on average: places of large tiles, beside runs of small tiles and empty ones
@pytest.mark.parametrize("heads,sizes", [(4, [0, 1, 24, 25, 30, 40, 64, 65]), (8, [0, 1, 4, 12, 13, 16, 17, 40]), (1, [0, 97, 96, 128, 129, 32, 257, 160])])
@pytest.mark.parametrize("count", [257, 300])
def test_many_chunks_of_large_tiles(fp8rl, heads, sizes, count):
    announce(f"chunk: {count} sequences, {heads} heads over one, runs of {sizes}")
    rng = np.random.default_rng(count + heads)
    new = rng.choice(sizes, count)
    assert new.mean() * heads > 86
    lens = new + rng.integers(0, 40, count)
    kc, vc, table = paged(rng, lens, 1)
    cu = offsets(new)
    q = bf16(rng, (int(cu[-1]), heads, 128))
    out = fp8rl.fp8rl_attention_prompt_fp8kv(q.cuda(), torch.from_numpy(kc).cuda(), torch.from_numpy(vc).cuda(), i32(table), i32(lens),
                                             i32(cu), int(lens.max()), f32_1(KS), f32_1(VS), SM)
    torch.cuda.synchronize()
    check(out, attention.prompt_paged(u16(q), kc, vc, KS, VS, table, lens, cu, SM), int(lens.max()), attention.FP8_VALUES, "chunk")


@pytest.mark.parametrize("sizes", [[0, 1, 11, 12, 13, 16, 17, 24], [12, 13]])
def test_many_groups_of_large_tiles(fp8rl, sizes):
    announce(f"shared: 280 groups of {sizes} members of 8 heads")
    rng = np.random.default_rng(len(sizes))
    count = 280
    members = rng.choice(sizes, count)
    go = offsets(members)
    batch = int(go[-1])
    assert members.mean() * 8 > 86
    lens = rng.integers(0, 120, batch)
    prefix = rng.integers(0, 110, count)
    kc, vc, table = paged(rng, lens, 1)
    q = bf16(rng, (batch, 8, 128))
    out = fp8rl.fp8rl_attention_decode_shared_fp8kv(
        q.cuda(), torch.from_numpy(kc).cuda(), torch.from_numpy(vc).cuda(), i32(table), i32(lens), i32(go), i32(prefix), 96, 120,
        f32_1(KS), f32_1(VS), SM)
    torch.cuda.synchronize()
    seen = attention.shared_table(table, lens, go, prefix, 96)
    check(out, attention.prompt_paged(u16(q), kc, vc, KS, VS, seen, lens, np.arange(batch + 1), SM), 120, attention.FP8_VALUES, "shared")


# (64 sequences a probe: 4096 take two levels of the search, more of them three)
@pytest.mark.parametrize("count", [4096, 4097, 5000])
def test_thousands_of_sequences(fp8rl, count):
    announce(f"prompt, chunk and shared: {count} sequences or groups of one token or so")
    rng = np.random.default_rng(count)
    lengths = rng.choice([0, 1, 2], count, p=[0.1, 0.8, 0.1])
    lengths[-1] = 1
    cu = offsets(lengths)
    n = int(cu[-1])
    q, k, v = bf16(rng, (n, 2, 128)), bf16(rng, (n, 1, 128)), bf16(rng, (n, 1, 128))
    out = fp8rl.fp8rl_attention_prompt_bf16(q.cuda(), k.cuda(), v.cuda(), i32(cu), 0.09)
    lens = lengths + rng.integers(0, 20, count)
    kc, vc, table = paged(rng, lens, 1)
    gkc, gvc, scales = torch.from_numpy(kc).cuda(), torch.from_numpy(vc).cuda(), (f32_1(KS), f32_1(VS))
    chunk = fp8rl.fp8rl_attention_prompt_fp8kv(q.cuda(), gkc, gvc, i32(table), i32(lens), i32(cu), 22, *scales, SM)
    prefix = np.minimum(lens, rng.integers(0, 20, count))
    q2 = bf16(rng, (count, 2, 128))
    shared = fp8rl.fp8rl_attention_decode_shared_fp8kv(q2.cuda(), gkc, gvc, i32(table), i32(lens), i32(np.arange(count + 1)), i32(prefix),
                                                       19, 22, *scales, SM)
    torch.cuda.synchronize()
    check(out, attention.prompt(u16(q), u16(k), u16(v), cu, 0.09), 2, attention.BF16_VALUES, "prompt")
    check(chunk, attention.prompt_paged(u16(q), kc, vc, KS, VS, table, lens, cu, SM), 22, attention.FP8_VALUES, "chunk")
    check(shared, attention.prompt_paged(u16(q2), kc, vc, KS, VS, table, lens, np.arange(count + 1), SM), 22, attention.FP8_VALUES,
          "shared")
