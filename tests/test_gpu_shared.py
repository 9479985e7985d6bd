"""Decode attention of sequences that share prefixes, against the fp64 oracle over the table that a group's sequences
see, within oracle.attention.bound."""
import numpy as np
import pytest
import torch

from oracle import attention
from tests.attn_util import bf16, check, f32_1, i32, offsets, paged, same
from tests.gpu_util import announce, need_gpu, u16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fp8rl():
    need_gpu()
    import paper_2601_18150_amd as m
    m.load()
    return m


def run(fp8rl, q, kc, vc, table, lens, go, prefix, max_prefix, max_len, sm=0.02, **kw):
    batch, heads = q.shape[:2]
    need = fp8rl.fp8rl_attention_decode_shared_workspace_size(batch, len(prefix), heads, kc.shape[1], max_prefix, max_len)
    ws = torch.full((max(need, 16) // 4,), float("nan"), dtype=torch.float32, device="cuda")
    out = fp8rl.fp8rl_attention_decode_shared_fp8kv(
        q.cuda(), torch.from_numpy(kc).cuda(), torch.from_numpy(vc).cuda(), i32(table), i32(lens), i32(go), i32(prefix),
        max_prefix, max_len, f32_1(0.02), f32_1(0.03), sm, workspace=ws, **kw)
    torch.cuda.synchronize()
    return out


def reference(q, kc, vc, table, lens, go, prefix, max_prefix, max_len, sm=0.02):
    lens = np.clip(lens, 0, max_len)
    seen = attention.shared_table(table, lens, go, prefix, max_prefix)
    return attention.prompt_paged(u16(q), kc, vc, np.float32(0.02), np.float32(0.03), seen, lens,
                                  np.arange(len(lens) + 1), sm)


def both(fp8rl, rng, heads, kv_heads, lens, go, prefix, max_prefix=None, max_len=None):
    max_prefix = max(list(prefix) + [0]) if max_prefix is None else max_prefix
    max_len = max(max(lens), max_prefix) if max_len is None else max_len
    kc, vc, table = paged(rng, lens, kv_heads, extra_pages=max(0, (max_len + 15) // 16 - (max(max(lens), 1) + 15) // 16))
    # (the other members' entries for the shared pages name blocks of their own, or none: they are not read)
    q = bf16(rng, (len(lens), heads, 128))
    out = run(fp8rl, q, kc, vc, table, lens, go, prefix, max_prefix, max_len)
    check(out, reference(q, kc, vc, table, lens, go, prefix, max_prefix, max_len), max_len, attention.FP8_VALUES, "shared")
    same(out, run(fp8rl, q, kc, vc, table, lens, go, prefix, max_prefix, max_len), "not deterministic")
    return out


@pytest.mark.parametrize("heads,kv_heads", [(3, 3), (4, 2), (8, 2), (16, 2)])
@pytest.mark.parametrize("lens,go,prefix", [
    ([50], [0, 1], [32]),
    ([48, 65, 33], [0, 3], [32]),                              # a member one token behind the prefix
    ([32, 32, 40], [0, 3], [32]),                              # members that are the prefix and nothing else
    ([100, 20, 0, 37, 90], [0, 3, 5], [64, 30]),               # shorter than the prefix, empty, a prefix inside a page
    ([20, 300, 5, 280, 7], [0, 2, 2, 4], [300, 64, 512]),      # a first member shorter than the prefix; an empty group;
                                                               # the last sequence in no group
    ([0, 90, 120], [0, 3], [80]),                              # an empty first member: nothing is shared
    ([15, 15], [0, 2], [15]),                                  # no whole page
])
def test_groups(fp8rl, heads, kv_heads, lens, go, prefix):
    announce(f"shared {heads}/{kv_heads} heads, lengths {lens}, groups {go}, prefixes {prefix}")
    out = both(fp8rl, np.random.default_rng(heads + len(lens)), heads, kv_heads, lens, go, prefix)
    assert torch.all(out[torch.tensor(lens) == 0] == 0)


def test_sequences_in_front_of_the_groups(fp8rl):
    announce("shared: sequences outside the groups on both sides")
    both(fp8rl, np.random.default_rng(1), 4, 1, [70, 70, 90, 33], [1, 3], [64])


# rows of a group past one tile (128), prefixes and own parts of several records
@pytest.mark.parametrize("heads,kv_heads,members,prefix,own", [(16, 2, 21, 700, 90), (4, 4, 130, 64, 40), (8, 1, 5, 5000, 3000)])
def test_large_groups(fp8rl, heads, kv_heads, members, prefix, own):
    announce(f"shared {heads}/{kv_heads} heads, {members} members, prefix {prefix}")
    rng = np.random.default_rng(members)
    prefix = prefix // 16 * 16
    lens = [prefix + int(n) for n in rng.integers(0, own + 1, members)]
    # the members' tables name the first one's blocks, as after a fork
    need = [prefix // 16] + [(n - prefix + 15) // 16 for n in lens]
    kc, vc, pages_of = paged(rng, [16 * n for n in need], kv_heads)
    table = np.full((members, (prefix + own + 15) // 16), -1, np.int32)
    table[:, :need[0]] = pages_of[0, :need[0]]
    for b in range(members):
        table[b, need[0]:need[0] + need[b + 1]] = pages_of[b + 1, :need[b + 1]]
    q = bf16(rng, (members, heads, 128))
    args = (q, kc, vc, table, lens, [0, members], [prefix], prefix, prefix + own)
    out = run(fp8rl, *args)
    check(out, reference(*args), prefix + own, attention.FP8_VALUES, "shared")
    alone = fp8rl.fp8rl_attention_decode_fp8kv(q.cuda(), torch.from_numpy(kc).cuda(), torch.from_numpy(vc).cuda(),
                                               i32(table), i32(lens), prefix + own, f32_1(0.02), f32_1(0.03), 0.02)
    torch.cuda.synchronize()
    check(alone, reference(*args), prefix + own, attention.FP8_VALUES, "each on its own")


def test_bounds_of_lengths(fp8rl):
    """Lengths above max_seq_len and prefixes above max_prefix_len count as those."""
    announce("shared: lengths above the bounds")
    both(fp8rl, np.random.default_rng(2), 4, 2, [200, 230, 150], [0, 3], [150], max_prefix=100, max_len=170)


def test_many_groups(fp8rl):
    """More groups than a wave has lanes, one or two sequences each."""
    announce("shared: 150 groups")
    rng = np.random.default_rng(3)
    sizes = rng.integers(0, 3, 150)
    go = offsets(sizes)
    lens = rng.integers(0, 60, int(go[-1])).tolist()
    both(fp8rl, rng, 2, 1, lens, go, rng.integers(0, 60, 150).tolist())


def test_captured_and_replayed(fp8rl):
    announce("shared: captured graph")
    rng = np.random.default_rng(4)
    lens, go, prefix = [700, 650, 800], [0, 3], [640]
    kc, vc, table = paged(rng, lens, 2)
    q = bf16(rng, (3, 8, 128)).cuda()
    args = [torch.from_numpy(kc).cuda(), torch.from_numpy(vc).cuda(), i32(table), i32(lens), i32(go), i32(prefix), 640, 800,
            f32_1(0.02), f32_1(0.03), 0.02]
    ws = torch.empty(fp8rl.fp8rl_attention_decode_shared_workspace_size(3, 1, 8, 2, 640, 800), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    fp8rl.fp8rl_attention_decode_shared_fp8kv(q, *args, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fp8rl.fp8rl_attention_decode_shared_fp8kv(q, *args, out=out, workspace=ws)
    for i in range(4):
        q.copy_(bf16(rng, (3, 8, 128)))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        want = fp8rl.fp8rl_attention_decode_shared_fp8kv(q, *args)
        torch.cuda.synchronize()
        same(got, want, f"replay {i}")
