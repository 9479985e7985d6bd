"""Attention against the cache where it changes its way: rows on both sides of a tile, shares of pages that end inside a
chunk of keys, caches past 4 GiB, streams other than the current one, two calls at once."""
import numpy as np
import pytest
import torch

from oracle import attention
from tests.attn_util import bf16, check, f32_1, i32, offsets, paged, same
from tests.gpu_util import announce, need_gpu, u16

pytestmark = pytest.mark.gpu
KS, VS, SM = np.float32(0.02), np.float32(0.03), 0.02


@pytest.fixture(scope="module")
def fp8rl():
    need_gpu()
    import paper_2601_18150_amd as m
    m.load()
    return m


def chunk_args(kc, vc, table, lens, cu, max_len):
    return [torch.from_numpy(kc).cuda(), torch.from_numpy(vc).cuda(), i32(table), i32(lens), i32(cu), max_len, f32_1(KS),
            f32_1(VS), SM]


# rows of a run: 32 a small tile, up to 96 in small tiles, 128 a large one
@pytest.mark.parametrize("heads,new", [(1, 31), (1, 32), (1, 33), (1, 64), (1, 65), (1, 96), (1, 97), (1, 128), (1, 129), (4, 8), (4, 9), (4, 16),
                                       (4, 17), (8, 8), (8, 9), (8, 12), (8, 13), (8, 33)])
def test_rows_at_the_edges_of_tiles(fp8rl, heads, new):
    announce(f"chunk: {heads} heads over one, {new} new tokens")
    rng = np.random.default_rng(heads * 1000 + new)
    lens, news = [new + 150, new, 77], [new, new, 1]
    kc, vc, table = paged(rng, lens, 1)
    cu = offsets(news)
    q = bf16(rng, (sum(news), heads, 128))
    out = fp8rl.fp8rl_attention_prompt_fp8kv(q.cuda(), *chunk_args(kc, vc, table, lens, cu, max(lens)))
    torch.cuda.synchronize()
    check(out, attention.prompt_paged(u16(q), kc, vc, KS, VS, table, lens, cu, SM), max(lens), attention.FP8_VALUES, "chunk")


# shares of a sequence's own pages that are no whole number of 32-key chunks, and the last one partly filled
@pytest.mark.parametrize("own", [1, 31, 255, 256, 257, 500, 528, 545, 815, 1100, 2049])
def test_shares_of_pages(fp8rl, own):
    announce(f"shared: {own} own tokens behind a prefix of 48")
    rng = np.random.default_rng(own)
    lens = [48 + own, 48 + max(1, own // 3)]
    kc, vc, table = paged(rng, lens, 1)
    table[1, :3] = table[0, :3]
    q = bf16(rng, (2, 4, 128))
    out = fp8rl.fp8rl_attention_decode_shared_fp8kv(
        q.cuda(), torch.from_numpy(kc).cuda(), torch.from_numpy(vc).cuda(), i32(table), i32(lens), i32([0, 2]), i32([48]), 48,
        max(lens), f32_1(KS), f32_1(VS), SM)
    torch.cuda.synchronize()
    check(out, attention.prompt_paged(u16(q), kc, vc, KS, VS, table, lens, [0, 1, 2], SM), max(lens), attention.FP8_VALUES,
          "shared")


def test_caches_past_4_gib(fp8rl):
    """Blocks spread over 4.6 GB of keys and of values: offsets of pages, chunks and copies past 32 bits."""
    announce("caches of 280000 blocks x 8 kv heads")
    rng = np.random.default_rng(1)
    lens = [300, 90, 1000]
    kc, vc, table = paged(rng, lens, 8)
    blocks = 280000
    at = np.sort(rng.choice(np.arange(200000, blocks), len(kc), replace=False))
    at[0], at[-1] = 0, blocks - 1
    ids = torch.from_numpy(at).cuda()
    big_k = torch.zeros((blocks, 8, 16, 128), dtype=torch.uint8, device="cuda")
    big_v = torch.zeros((blocks, 8, 4, 128, 4), dtype=torch.uint8, device="cuda")
    big_k[ids], big_v[ids] = torch.from_numpy(kc).cuda(), torch.from_numpy(vc).cuda()
    used = np.arange(table.shape[1])[None] < (np.array(lens)[:, None] + 15) // 16
    far = np.where(used, at[np.clip(table, 0, len(at) - 1)], -1).astype(np.int32)
    new = [40, 3, 1]                                     # large tiles, small ones
    cu = offsets(new)
    q = bf16(rng, (44, 16, 128))
    out = fp8rl.fp8rl_attention_prompt_fp8kv(q.cuda(), big_k, big_v, i32(far), i32(lens), i32(cu), 1000, f32_1(KS), f32_1(VS), SM)
    torch.cuda.synchronize()
    check(out, attention.prompt_paged(u16(q), kc, vc, KS, VS, table, lens, cu, SM), 1000, attention.FP8_VALUES, "chunk")
    q = bf16(rng, (3, 16, 128))
    out = fp8rl.fp8rl_attention_decode_shared_fp8kv(q.cuda(), big_k, big_v, i32(far), i32(lens), i32([0, 2, 3]), i32([80, 512]),
                                                    512, 1000, f32_1(KS), f32_1(VS), SM)
    torch.cuda.synchronize()
    seen = attention.shared_table(table, lens, [0, 2, 3], [80, 512], 512)
    check(out, attention.prompt_paged(u16(q), kc, vc, KS, VS, seen, lens, np.arange(4), SM), 1000, attention.FP8_VALUES, "shared")
    announce("copy and compact of the same")
    fp8rl.fp8rl_kv_copy_blocks([big_k, big_v], i32([at[-1]]), i32([blocks - 3]))
    torch.cuda.synchronize()
    assert torch.equal(big_k[blocks - 3], big_k[blocks - 1]) and torch.equal(big_v[blocks - 3], big_v[blocks - 1])
    refs = torch.zeros(blocks, dtype=torch.int32, device="cuda")
    refs[torch.from_numpy(far[used]).cuda().long()] = 1
    state = [i32(far), i32(lens), refs]
    live = fp8rl.fp8rl_kv_compact([big_k, big_v], *state)
    torch.cuda.synchronize()
    assert int(live) == used.sum() and torch.all(refs[:int(live)] == 1) and int(refs.sum()) == int(live)
    now = state[0].cpu().numpy()
    assert np.array_equal(big_k[torch.from_numpy(now[used]).cuda().long()].cpu().numpy(), kc[table[used]])
    assert np.array_equal(big_v[torch.from_numpy(now[used]).cuda().long()].cpu().numpy(), vc[table[used]])


def test_on_a_stream_of_its_own_and_two_at_once(fp8rl):
    """Inputs made on one stream, calls on two others without anything to order them but the events: each allocates its
    own workspace and output there."""
    announce("chunk and shared on side streams")
    rng = np.random.default_rng(2)
    lens, new = [3000, 700], [2, 40]
    kc, vc, table = paged(rng, lens, 2)
    cu = offsets(new)
    qs = [bf16(rng, (42, 8, 128)).cuda() for _ in range(6)]
    args = chunk_args(kc, vc, table, lens, cu, 3000)
    group = [i32([0, 2]), i32([640]), 640, 3000]

    def both(q, stream=None):
        a = fp8rl.fp8rl_attention_prompt_fp8kv(q, *args, stream=stream)
        b = fp8rl.fp8rl_attention_decode_shared_fp8kv(q[:2], *args[:4], *group, *args[6:], stream=stream)
        return a, b

    want = [both(q) for q in qs]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [both(q, streams[i % 2]) for i, q in enumerate(qs)]
    by_handle = both(qs[0], streams[0].cuda_stream)
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        same(g[0], w[0], "chunk on a side stream")
        same(g[1], w[1], "shared on a side stream")
    same(by_handle[0], want[0][0], "chunk on a stream by its handle")
    same(by_handle[1], want[0][1], "shared on a stream by its handle")


def finite_alone(got, res, clean, keys, kind, what):
    """Where the oracle is finite the outputs are within the bound of the same inputs without the values that are not
    (`clean`: a row that sees them has other dims of which they are no part); elsewhere they are the oracle's."""
    g = got.float().cpu().numpy().astype(np.float64).reshape(res[0].shape)
    ok = np.isfinite(res[0])
    assert not ok.all() and ok.any()
    assert np.array_equal(g[~ok], res[0][~ok], equal_nan=True), f"{what}: not the oracle's where it is not finite"
    check(torch.from_numpy(np.where(ok, g, np.nan)), (np.where(ok, clean[0], np.nan), *clean[1:]), keys, kind, what)


# (up to 512 workgroups take tiles of 64 rows, more of them ones of 128)
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 1), (4, 2), (180, 180)])
@pytest.mark.parametrize("at", [0, 40, 100, 149])
def test_values_that_are_not_finite_reach_later_prompt_rows_alone(fp8rl, heads, kv_heads, at):
    announce(f"prompt: {heads}/{kv_heads} heads, NaN and inf among the values of token {at}, a NaN key behind it")
    rng = np.random.default_rng(heads + at)
    n = 200
    cu = [0, n, n + 30]
    q, k, v = bf16(rng, (n + 30, heads, 128)), bf16(rng, (n + 30, kv_heads, 128)), bf16(rng, (n + 30, kv_heads, 128))
    clean = attention.prompt(u16(q), u16(k), u16(v), cu, 0.09)
    v[at, 0, 5], v[at, kv_heads - 1, 77], v[at + 1, 0, 9], k[at + 30, 0, 3] = float("nan"), float("inf"), -float("inf"), float("nan")
    with np.errstate(invalid="ignore"):
        res = attention.prompt(u16(q), u16(k), u16(v), cu, 0.09)
    out = fp8rl.fp8rl_attention_prompt_bf16(q.cuda(), k.cuda(), v.cuda(), i32(cu), 0.09)
    torch.cuda.synchronize()
    finite_alone(out, res, clean, n, attention.BF16_VALUES, "prompt")


def poison(vc, table, b, token, dim):
    vc[table[b, token // 16], :, token % 16 // 4, dim, token % 4] = 0x7F


# small tiles and large ones, whole and in records
@pytest.mark.parametrize("heads,kv_heads,lens,new", [(2, 1, [150, 40], [20, 5]), (8, 1, [150, 170], [40, 3]),
                                                     (4, 1, [3000, 700], [6, 20]), (8, 2, [1500, 2100], [33, 70])])
def test_nan_codes_of_later_tokens_do_not_reach_a_chunk(fp8rl, heads, kv_heads, lens, new):
    announce(f"chunk: {heads}/{kv_heads} heads, lengths {lens}, new {new}, NaN codes among the new tokens' values")
    rng = np.random.default_rng(heads + new[0])
    kc, vc, table = paged(rng, lens, kv_heads)
    cu = offsets(new)
    q = bf16(rng, (sum(new), heads, 128))
    args = [u16(q), kc, vc, KS, VS, table, lens, cu, SM]
    clean = attention.prompt_paged(*args)
    for b, (n, m) in enumerate(zip(lens, new)):
        poison(vc, table, b, n - 1, 3)
        poison(vc, table, b, n - m // 2, 100)
    res = attention.prompt_paged(*args)
    out = fp8rl.fp8rl_attention_prompt_fp8kv(q.cuda(), *chunk_args(kc, vc, table, lens, cu, max(lens)))
    torch.cuda.synchronize()
    finite_alone(out, res, clean, max(lens), attention.FP8_VALUES, "chunk")


@pytest.mark.parametrize("heads,members", [(2, 5), (8, 40)])
def test_nan_codes_behind_a_short_member_do_not_reach_it(fp8rl, heads, members):
    """Members shorter than their prefix: what the others read behind their end is not theirs."""
    announce(f"shared: {members} members of {heads} heads, NaN codes in the prefix behind the short ones")
    rng = np.random.default_rng(members)
    lens = [900] + [int(x) for x in rng.integers(1, 900, members - 1)]
    kc, vc, table = paged(rng, [900] * members, 1)
    table[1:] = table[0]
    q = bf16(rng, (members, heads, 128))
    args = [u16(q), kc, vc, KS, VS, table, lens, np.arange(members + 1), SM]
    clean = attention.prompt_paged(*args)
    for t in (100, 333, 640, 890):
        poison(vc, table, 0, t, t % 128)
    res = attention.prompt_paged(*args)
    out = fp8rl.fp8rl_attention_decode_shared_fp8kv(
        q.cuda(), torch.from_numpy(kc).cuda(), torch.from_numpy(vc).cuda(), i32(table), i32(lens), i32([0, members]), i32([896]),
        896, 900, f32_1(KS), f32_1(VS), SM)
    torch.cuda.synchronize()
    finite_alone(out, res, clean, 900, attention.FP8_VALUES, "shared")


@pytest.mark.parametrize("new,length", [(3, 3), (40, 200), (2, 3000)])
def test_a_row_whose_scores_are_all_minus_infinity(fp8rl, new, length):
    """No softmax exists of them: NaN, whichever way the row takes; the rows beside it keep theirs."""
    announce(f"chunk and prompt: {new} of {length} tokens, one row of -inf scores")
    rng = np.random.default_rng(new)
    kc, vc, table = paged(rng, [length], 1)
    kc[:, :, :, 0] = 0x7E                                # 448 in dim 0 of every key
    q = bf16(rng, (new, 4, 128))
    q[:, :, 0] = 0.0
    res = attention.prompt_paged(u16(q), kc, vc, KS, VS, table, [length], [0, new], SM)
    q[1, 2, 0] = -3e38
    out = fp8rl.fp8rl_attention_prompt_fp8kv(q.cuda(), *chunk_args(kc, vc, table, [length], [0, new], length))
    k, v = torch.zeros((new, 1, 128), dtype=torch.bfloat16), bf16(rng, (new, 1, 128))
    k[:, :, 0] = 448.0
    prompt = fp8rl.fp8rl_attention_prompt_bf16(q.cuda(), k.cuda(), v.cuda(), i32([0, new]), SM)
    torch.cuda.synchronize()
    assert torch.isnan(out[1, 2]).all() and torch.isnan(prompt[1, 2]).all()
    out, prompt = out.clone(), prompt.clone()
    out[1, 2] = torch.from_numpy(res[0][1, 2]).to(out)
    prompt[1, 2] = 0.0
    check(out, res, length, attention.FP8_VALUES, "chunk")
    assert torch.isfinite(prompt).all()


@pytest.mark.parametrize("count", [255, 256, 257, 600])
def test_many_short_sequences(fp8rl, count):
    """The tiles' search looks at 256 sequences a step: counts on both sides of that, and more; none, one or more tiles each."""
    announce(f"chunk and shared: {count} sequences or groups")
    rng = np.random.default_rng(count)
    new = rng.choice([0, 1, 2, 40], count, p=[0.3, 0.4, 0.28, 0.02])
    new[-1] = 3
    lens = new + rng.integers(0, 20, count)
    kc, vc, table = paged(rng, lens, 1)
    cu = offsets(new)
    q = bf16(rng, (int(cu[-1]), 4, 128))
    out = fp8rl.fp8rl_attention_prompt_fp8kv(q.cuda(), *chunk_args(kc, vc, table, lens, cu, int(lens.max())))
    sizes = rng.integers(0, 3, count)
    sizes[0], sizes[-1] = 1, 2
    go = offsets(sizes)
    lens2 = rng.integers(0, 50, int(go[-1]))
    prefix = rng.integers(0, 50, count)
    kc2, vc2, table2 = paged(rng, lens2, 1)
    q2 = bf16(rng, (int(go[-1]), 4, 128))
    shared = fp8rl.fp8rl_attention_decode_shared_fp8kv(
        q2.cuda(), torch.from_numpy(kc2).cuda(), torch.from_numpy(vc2).cuda(), i32(table2), i32(lens2), i32(go), i32(prefix),
        48, 50, f32_1(KS), f32_1(VS), SM)
    torch.cuda.synchronize()
    check(out, attention.prompt_paged(u16(q), kc, vc, KS, VS, table, lens, cu, SM), 60, attention.FP8_VALUES, "chunk")
    seen = attention.shared_table(table2, lens2, go, prefix, 48)
    check(shared, attention.prompt_paged(u16(q2), kc2, vc2, KS, VS, seen, lens2, np.arange(len(lens2) + 1), SM), 50,
          attention.FP8_VALUES, "shared")


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 1), (4, 2)])
def test_many_prompts(fp8rl, heads, kv_heads):
    """More prompts than are counted one by one: empty ones, whole tiles, a few long ones, rows in front and behind."""
    announce(f"prompt: 400 sequences, {heads}/{kv_heads} heads")
    rng = np.random.default_rng(heads)
    lengths = rng.choice([0, 1, 16, 32, 33, 300], 400, p=[0.3, 0.3, 0.19, 0.1, 0.1, 0.01])
    cu = offsets(lengths, 3)
    n = int(cu[-1]) + 5
    q, k, v = bf16(rng, (n, heads, 128)), bf16(rng, (n, kv_heads, 128)), bf16(rng, (n, kv_heads, 128))
    out = torch.full((n, heads, 128), 9.0, dtype=torch.bfloat16, device="cuda")
    fp8rl.fp8rl_attention_prompt_bf16(q.cuda(), k.cuda(), v.cuda(), i32(cu), 0.09, out=out)
    torch.cuda.synchronize()
    check(out, attention.prompt(u16(q), u16(k), u16(v), cu, 0.09), 300, attention.BF16_VALUES, "prompt")
    assert torch.all(out[:3] == 9.0) and torch.all(out[int(cu[-1]):] == 9.0)


@pytest.mark.parametrize("go,prefix,max_prefix", [([0, 3], [64], 0), ([1, 1, 1], [64, 64], 64), ([0, 3], [-5], 64), ([3, 3], [64], 64)])
def test_nothing_shared(fp8rl, go, prefix, max_prefix):
    announce(f"shared: groups {go}, prefixes {prefix}, at most {max_prefix}; a negative length")
    rng = np.random.default_rng(5)
    lens = [90, 33, 70]
    kc, vc, table = paged(rng, lens, 2)
    q = bf16(rng, (3, 4, 128))
    out = fp8rl.fp8rl_attention_decode_shared_fp8kv(
        q.cuda(), torch.from_numpy(kc).cuda(), torch.from_numpy(vc).cuda(), i32(table), i32([90, -7, 70]), i32(go), i32(prefix),
        max_prefix, 90, f32_1(KS), f32_1(VS), SM)
    chunk = fp8rl.fp8rl_attention_prompt_fp8kv(q.cuda(), *chunk_args(kc, vc, table, [90, -7, 70], [0, 1, 2, 3], 90))
    torch.cuda.synchronize()
    res = attention.prompt_paged(u16(q), kc, vc, KS, VS, table, [90, 0, 70], [0, 1, 2, 3], SM)
    check(out, res, 90, attention.FP8_VALUES, "shared")
    check(chunk, res, 90, attention.FP8_VALUES, "chunk")
    assert torch.all(out[1] == 0) and torch.all(chunk[1] == 0)


@pytest.mark.parametrize("group", [1, 2, 4, 8])
@pytest.mark.parametrize("lengths", [[1, 15, 16, 17], [31, 33, 0, 65], [129], [200, 7]])
def test_prompts_of_many_heads(fp8rl, group, lengths):
    """More than 512 workgroups, which take tiles of 128 rows, and few, which take ones of 64."""
    announce(f"prompt: 520 kv heads, {group} query heads each, lengths {lengths}")
    rng = np.random.default_rng(group + len(lengths))
    cu, n = offsets(lengths), sum(lengths)
    q, k, v = bf16(rng, (n, 520 * group, 128)), bf16(rng, (n, 520, 128)), bf16(rng, (n, 520, 128))
    out = fp8rl.fp8rl_attention_prompt_bf16(q.cuda(), k.cuda(), v.cuda(), i32(cu), 0.09)
    torch.cuda.synchronize()
    some = [0, 1, 269, 518, 519]                             # (the oracle's time: five of the kv heads)
    heads = [h * group + g for h in some for g in range(group)]
    check(out[:, heads], attention.prompt(u16(q[:, heads]), u16(k[:, some]), u16(v[:, some]), cu, 0.09), 200,
          attention.BF16_VALUES, "prompt")
    few = fp8rl.fp8rl_attention_prompt_bf16(q[:, heads].cuda(), k[:, some].cuda(), v[:, some].cuda(), i32(cu), 0.09)
    torch.cuda.synchronize()
    check(few, attention.prompt(u16(q[:, heads]), u16(k[:, some]), u16(v[:, some]), cu, 0.09), 200, attention.BF16_VALUES, "few heads")
