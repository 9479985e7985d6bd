"""Pages of the cache: copies, forks, frees and compactions against the page oracle, every byte and count; and a
rollout's life of a cache through all the operators that work on it."""
import numpy as np
import pytest
import torch

from oracle import attention, pages
from tests.attn_util import bf16, check, f32_1, i32, offsets
from tests.gpu_util import announce, need_gpu, u16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fp8rl():
    need_gpu()
    import paper_2601_18150_amd as m
    m.load()
    return m


def pool(rng, count, blocks, block_bytes):
    return [rng.integers(0, 256, (blocks, block_bytes)).astype(np.uint8) for _ in range(count)]


def to_gpu(arrays):
    return [torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in arrays]


def assert_same(gpu, host, what):
    torch.cuda.synchronize()
    for i, (g, h) in enumerate(zip(gpu, host)):
        assert np.array_equal(g.cpu().numpy(), h), f"{what} {i}"


# block sizes on both sides of a workgroup's 16 KiB step; more caches than one launch takes
@pytest.mark.parametrize("caches,blocks,block_bytes", [(1, 9, 16), (2, 40, 2048), (3, 20, 16384), (2, 8, 40016), (131, 12, 64)])
def test_copy_blocks(fp8rl, caches, blocks, block_bytes):
    announce(f"copy blocks: {caches} caches of {blocks} x {block_bytes}")
    rng = np.random.default_rng(caches)
    host = pool(rng, caches, blocks, block_bytes)
    gpu = to_gpu(host)
    perm = rng.permutation(blocks)
    n = blocks // 2
    src, dst = perm[:n].astype(np.int32), perm[n:2 * n].astype(np.int32)
    src[0], dst[-1] = -1, blocks                          # skipped
    fp8rl.fp8rl_kv_copy_blocks(gpu, i32(src), i32(dst))
    pages.copy_blocks(host, src, dst)
    assert_same(gpu, host, "cache")


def sequences(rng, lens, rows, max_blocks, blocks):
    """Rows 0 .. of the given lengths over shuffled blocks: (table, lens, refs, the free blocks)."""
    table = rng.integers(-3, blocks + 3, (rows, max_blocks)).astype(np.int32)   # (anything behind a row's length)
    full, refs, free = np.zeros(rows, np.int32), np.zeros(blocks, np.int32), list(rng.permutation(blocks))
    for r, n in enumerate(lens):
        used = (n + 15) // 16
        table[r, :used], full[r] = free[:used], n
        refs[free[:used]] += 1
        free = free[used:]
    return table, full, refs, free


@pytest.mark.parametrize("caches", [1, 5, 130])
def test_fork_and_free(fp8rl, caches):
    """Whole and partly filled last pages, an empty parent, a parent of a full row, forks that are skipped."""
    announce(f"fork and free: {caches} caches")
    rng = np.random.default_rng(caches + 1)
    lens = [33, 16, 0, 96, 95, 1]
    table, full, refs, free = sequences(rng, lens, 20, 6, 60)
    host = pool(rng, caches, 60, 4096)
    gpu, state = to_gpu(host), to_gpu([table, full, refs])
    parents = [0, 0, 1, 2, 3, 4, 5, 0, 1, 20, -1, 4, 5, 6]
    children = [6, 7, 8, 9, 10, 11, 12, 20, -2, 13, 14, 15, 16, 6]
    new = [int(b) for b in free[:11]] + [-1, 60, int(free[11])]   # no block: skipped; a row to itself (6, 6): skipped
    fp8rl.fp8rl_kv_fork_sequences(gpu, *state, i32(parents[:13] + [7]), i32(children[:13] + [7]), i32(new))
    pages.fork(host, table, full, refs, parents[:13] + [7], children[:13] + [7], new)
    assert_same(gpu, host, "cache")
    assert_same(state, [table, full, refs], "table, lengths, counts:")
    gone = [0, 6, 6, 11, 3, -1, 99, 2]
    fp8rl.fp8rl_kv_free_sequences(*state, i32(gone))
    pages.free(table, full, refs, gone)
    assert_same(state, [table, full, refs], "table, lengths, counts:")


# chunks of 2048 blocks: one, a whole number, a ragged one
@pytest.mark.parametrize("blocks,share", [(1, 0.0), (1, 1.0), (50, 0.5), (50, 0.0), (50, 1.0), (2048, 0.3), (2049, 0.9),
                                          (10000, 0.02), (10000, 0.6)])
def test_compact(fp8rl, blocks, share):
    announce(f"compact: {blocks} blocks, {share} of them in use")
    rng = np.random.default_rng(blocks)
    refs = np.where(rng.random(blocks) < share, rng.integers(1, 4, blocks), rng.integers(-1, 1, blocks)).astype(np.int32)
    used = np.flatnonzero(refs > 0)
    rows, width = 7, 40
    table = rng.integers(-2, blocks + 2, (rows, width)).astype(np.int32)
    if len(used):
        table[:, ::2] = rng.choice(used, (rows, (width + 1) // 2))
    lens = rng.integers(0, width * 16 + 40, rows).astype(np.int32)   # (past the row: counts as the row's end)
    host = pool(rng, 3, blocks, 48)
    gpu, state = to_gpu(host), to_gpu([table, lens, refs])
    live = fp8rl.fp8rl_kv_compact(gpu, *state)
    want = pages.compact(host, table, lens, refs)
    assert_same([live], [np.array([want], np.int32)], "blocks in use")
    assert_same(gpu, host, "cache")
    # (a count at or below 0 marks a free block; the ones below L that were free hold a mover's count now)
    assert_same(state, [table, lens, refs], "table, lengths, counts:")
    again = fp8rl.fp8rl_kv_compact(gpu, *state)
    assert_same(gpu + state + [again], host + [table, lens, refs, np.array([want], np.int32)], "a second time")


def test_compact_many_caches_and_rows(fp8rl):
    announce("compact: 140 caches, 3000 rows")
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 30, 3000).tolist()
    table, full, refs, _ = sequences(rng, lens, 3000, 2, 6000)
    host = pool(rng, 140, 6000, 16)
    gone = rng.permutation(3000)[:2000]
    pages.free(table, full, refs, gone)
    gpu, state = to_gpu(host), to_gpu([table, full, refs])
    fp8rl.fp8rl_kv_compact(gpu, *state)
    pages.compact(host, table, full, refs)
    assert_same(gpu, host, "cache")
    assert_same(state, [table, full, refs], "table, lengths, counts:")


def test_captured_and_replayed(fp8rl):
    """Fork, free and compact in one graph: every replay, on tables put back before it, gives the same state."""
    announce("pages: captured graph")
    rng = np.random.default_rng(6)
    table, full, refs, free = sequences(rng, [40, 100, 7], 8, 8, 64)
    host = pool(rng, 4, 64, 2048)
    gpu, first, state = to_gpu(host), to_gpu([table, full, refs]), to_gpu([table, full, refs])
    start = [g.clone() for g in gpu]
    live, ws = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.empty(
        fp8rl.fp8rl_kv_compact_workspace_size(64), dtype=torch.uint8, device="cuda")
    job = [i32([0, 1, 2]), i32([3, 4, 5]), i32(free[:3])]
    gone = i32([0, 1])

    def step():
        fp8rl.fp8rl_kv_fork_sequences(gpu, *state, *job)
        fp8rl.fp8rl_kv_free_sequences(*state, gone)
        fp8rl.fp8rl_kv_compact(gpu, *state, live=live, workspace=ws)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    pages.fork(host, table, full, refs, [0, 1, 2], [3, 4, 5], free[:3])
    pages.free(table, full, refs, [0, 1])
    want = pages.compact(host, table, full, refs)
    for i in range(4):
        for now, x in zip(gpu + state, start + first):
            now.copy_(x)
        graph.replay()
        assert_same(gpu + state + [live], host + [table, full, refs, np.array([want], np.int32)], f"replay {i}:")


def test_rollout_of_two_prompts(fp8rl):
    """Prompts through attention and into the cache, forked to samples, a decode step of all samples with the prompts'
    pages read once, half of the samples freed, the cache compacted, and the next step of those left."""
    announce("rollout: prompt, write, fork, shared decode, free, compact, shared decode")
    rng = np.random.default_rng(7)
    heads, kv_heads, samples, sm = 8, 2, 5, float(1 / np.sqrt(128))
    prompts = [70, 33]
    cu = offsets(prompts)
    q, k, v = bf16(rng, (103, heads, 128)), bf16(rng, (103, kv_heads, 128)), bf16(rng, (103, kv_heads, 128))
    out = fp8rl.fp8rl_attention_prompt_bf16(q.cuda(), k.cuda(), v.cuda(), i32(cu), sm)
    check(out, attention.prompt(u16(q), u16(k), u16(v), cu, sm), 70, attention.BF16_VALUES, "prompt")

    blocks, rows, width = 64, 2 + 2 * samples, 8
    table, lens, refs, free = sequences(rng, prompts, rows, width, blocks)
    kc, vc = (torch.zeros((blocks, kv_heads) + s, dtype=torch.uint8, device="cuda") for s in ((16, 128), (4, 128, 4)))
    ks, vs = fp8rl.fp8rl_kv_calibrate_scale(k.cuda()), fp8rl.fp8rl_kv_calibrate_scale(v.cuda())
    slots = torch.from_numpy(np.concatenate([table[b, np.arange(n) // 16].astype(np.int64) * 16 + np.arange(n) % 16
                                             for b, n in enumerate(prompts)])).cuda()
    fp8rl.fp8rl_kv_cache_write_fp8(k.cuda(), v.cuda(), slots, ks, vs, kc, vc)
    cached = fp8rl.fp8rl_attention_prompt_fp8kv(q.cuda(), kc, vc, i32(table[:2]), i32(prompts), i32(cu), 70, ks, vs, sm)
    res = attention.prompt_paged(u16(q), kc.cpu().numpy(), vc.cpu().numpy(), ks.item(), vs.item(), table, prompts, cu, sm)
    check(cached, res, 70, attention.FP8_VALUES, "prompt against the cache")

    state = to_gpu([table, lens, refs])
    children = list(range(2, rows))
    fp8rl.fp8rl_kv_fork_sequences([kc, vc], *state, i32([0] * samples + [1] * samples), i32(children), i32(free[:2 * samples]))
    fp8rl.fp8rl_kv_free_sequences(*state, i32([0, 1]))     # the prompts' own rows end; their pages live on in the samples

    def step(rows_of, go, prefix):
        """A new token of each row (room for it is in its last page) and its attention."""
        rows_of = torch.tensor(rows_of, device="cuda")
        n = len(rows_of)
        qn, kn, vn = bf16(rng, (n, heads, 128)), bf16(rng, (n, kv_heads, 128)), bf16(rng, (n, kv_heads, 128))
        at = state[1][rows_of].long()
        slot = state[0][rows_of].gather(1, (at // 16)[:, None])[:, 0].long() * 16 + at % 16
        fp8rl.fp8rl_kv_cache_write_fp8(kn.cuda(), vn.cuda(), slot, ks, vs, kc, vc)
        state[1][rows_of] += 1
        t, ln = state[0][rows_of].contiguous(), state[1][rows_of].contiguous()
        got = fp8rl.fp8rl_attention_decode_shared_fp8kv(qn.cuda(), kc, vc, t, ln, i32(go), i32(prefix), 70, 80, ks, vs, sm)
        torch.cuda.synchronize()
        want = attention.prompt_paged(u16(qn), kc.cpu().numpy(), vc.cpu().numpy(), ks.item(), vs.item(), t.cpu().numpy(),
                                      ln.cpu().numpy(), np.arange(n + 1), sm)
        check(got, want, 80, attention.FP8_VALUES, f"decode of {n}")

    step(children, [0, samples, 2 * samples], prompts)
    fp8rl.fp8rl_kv_free_sequences(*state, i32(children[::2]))
    live = fp8rl.fp8rl_kv_compact([kc, vc], *state)
    torch.cuda.synchronize()
    # five samples left, three of prompt 1 (rows 7 + 1, ..): whole pages of both prompts and a page of each sample
    left = children[1::2]
    assert int(live) == 70 // 16 + 33 // 16 + len(left)
    step(left, [0, 2, 5], prompts)
