"""Causal attention over packed prompts and over chunks against the paged FP8 cache, against the fp64 oracle within
the bound that oracle.attention.bound derives from the kernel's roundings."""
import numpy as np
import pytest
import torch

from oracle import attention
from tests.attn_util import bf16, check, f32_1, i32, offsets, paged, same
from tests.gpu_util import announce, need_gpu, u16

pytestmark = pytest.mark.gpu
SM = float(1 / np.sqrt(128))


@pytest.fixture(scope="module")
def fp8rl():
    need_gpu()
    import paper_2601_18150_amd as m
    m.load()
    return m


def run_prompt(fp8rl, q, k, v, cu, sm=SM, **kw):
    out = fp8rl.fp8rl_attention_prompt_bf16(q.cuda(), k.cuda(), v.cuda(), i32(cu), sm, **kw)
    torch.cuda.synchronize()
    return out


# tiles hold 128 / group tokens and 64 keys: lengths on both sides of their edges, empty sequences among them
@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (6, 3), (8, 2), (16, 2)])
@pytest.mark.parametrize("lengths", [[1], [0, 1, 0, 2, 17, 0], [15, 16, 17, 31, 32, 33], [63, 64, 65], [127, 129], [300, 5, 200]])
def test_prompt_lengths_and_heads(fp8rl, heads, kv_heads, lengths):
    announce(f"prompt {heads}/{kv_heads} heads, lengths {lengths}")
    rng = np.random.default_rng(heads * 100 + len(lengths))
    n = sum(lengths)
    q, k, v = (bf16(rng, (n, h, 128)) for h in (heads, kv_heads, kv_heads))
    cu = offsets(lengths)
    out = run_prompt(fp8rl, q, k, v, cu)
    check(out, attention.prompt(u16(q), u16(k), u16(v), cu, SM), max(lengths), attention.BF16_VALUES, "prompt")
    same(out, run_prompt(fp8rl, q, k, v, cu), "not deterministic")


def test_prompt_of_many_tiles(fp8rl):
    announce("prompt of 1500 tokens, 2 heads over 1")
    rng = np.random.default_rng(9)
    q, k, v = bf16(rng, (1500, 2, 128)), bf16(rng, (1500, 1, 128), 2.0), bf16(rng, (1500, 1, 128))
    check(run_prompt(fp8rl, q, k, v, [0, 1500]), attention.prompt(u16(q), u16(k), u16(v), [0, 1500], SM), 1500,
          attention.BF16_VALUES, "prompt")


def test_prompt_many_sequences(fp8rl):
    """More sequences than a wave has lanes, so that the search for a tile's sequence takes several steps."""
    announce("prompt: 200 sequences")
    rng = np.random.default_rng(10)
    lengths = rng.integers(0, 9, 200)
    cu, n = offsets(lengths), int(lengths.sum())
    q, k, v = bf16(rng, (n, 2, 128)), bf16(rng, (n, 2, 128)), bf16(rng, (n, 2, 128))
    check(run_prompt(fp8rl, q, k, v, cu), attention.prompt(u16(q), u16(k), u16(v), cu, SM), 8, attention.BF16_VALUES, "prompt")


def test_prompt_from_a_fused_output_into_a_padded_one(fp8rl):
    """q, k, v as column ranges of one matrix with a row pitch of its own; rows of no sequence (in front, behind) hold
    NaN, which no row may see, and stay as they are in the output."""
    announce("prompt: fused qkv, padded rows, NaN outside")
    rng = np.random.default_rng(11)
    heads, kv_heads, total = 8, 2, 150
    cu = offsets([37, 0, 90], 4)
    fused = bf16(rng, (total, 12 * 128 + 64))
    fused[:4], fused[131:] = float("nan"), float("nan")
    view = fused.cuda()[:, :12 * 128].view(total, 12, 128)
    out = torch.full((total, heads * 128 + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    rows = out[:, :heads * 128].view(total, heads, 128)
    fp8rl.fp8rl_attention_prompt_bf16(view[:, :8], view[:, 8:10], view[:, 10:], i32(cu), SM, out=rows)
    torch.cuda.synchronize()
    host = fused[:, :12 * 128].reshape(total, 12, 128)
    res = attention.prompt(u16(host[:, :8]), u16(host[:, 8:10]), u16(host[:, 10:]), cu, SM)
    check(rows, res, 90, attention.BF16_VALUES, "prompt")
    assert torch.all(rows[:4] == 7.0) and torch.all(rows[131:] == 7.0) and torch.all(out[:, heads * 128:] == 7.0)


def test_prompt_sees_nothing_of_the_call_before(fp8rl):
    """Rows behind a short sequence's end, inside its tiles, count as zeros whatever LDS held before (here NaN)."""
    announce("prompt: short sequences after a call with NaN everywhere")
    rng = np.random.default_rng(16)
    nan = torch.full((20000, 8, 128), float("nan"), dtype=torch.bfloat16)
    run_prompt(fp8rl, nan, nan, nan, [0, 20000])
    lengths = rng.integers(1, 40, 500)
    cu, n = offsets(lengths), int(lengths.sum())
    q, k, v = (bf16(rng, (n, 1, 128)) for _ in range(3))
    check(run_prompt(fp8rl, q, k, v, cu), attention.prompt(u16(q), u16(k), u16(v), cu, SM), 40, attention.BF16_VALUES, "prompt")


@pytest.mark.parametrize("sm", [1e-38, 3.0, 40.0])
def test_prompt_extreme_factors(fp8rl, sm):
    """A factor that makes every weight 1, and ones that make each row all but one key's."""
    announce(f"prompt: factor {sm}")
    rng = np.random.default_rng(12)
    q, k, v = (bf16(rng, (150, 2, 128)) for _ in range(3))
    res = attention.prompt(u16(q), u16(k), u16(v), [0, 150], sm)
    check(run_prompt(fp8rl, q, k, v, [0, 150], sm), res, 150, attention.BF16_VALUES, "prompt")


def test_prompt_scores_past_the_range_of_fp32(fp8rl):
    """Keys whose scores overflow to -inf weigh nothing, alone in a tile too (the first 70 of 140)."""
    announce("prompt: -inf scores")
    rng = np.random.default_rng(13)
    q, k, v = (bf16(rng, (140, 1, 128)) for _ in range(3))
    q[:, :, 0], k[:, :, 0] = 3e38, 0.0
    k[1:70, :, 0] = -448.0                          # (key 0 keeps a finite score, the one of the first rows)
    res = attention.prompt(u16(q), u16(k), u16(v), [0, 140], SM)
    # scores of magnitude 1e39 do not occur in fp32: what is left is as exact as the finite ones
    rest = (res[0], res[1], np.minimum(res[2], 140.0), res[3])
    check(run_prompt(fp8rl, q, k, v, [0, 140]), rest, 140, attention.BF16_VALUES, "prompt")


def test_prompt_offsets_past_32_bits(fp8rl):
    """A row pitch near the largest allowed: 150 rows span 5 GB of each tensor."""
    announce("prompt: row pitch 2^24 - 8")
    rng = np.random.default_rng(14)
    pitch, n = (1 << 24) - 8, 150
    q, k, v = (bf16(rng, (n, 1, 128)) for _ in range(3))
    wide = [torch.empty(n * pitch, dtype=torch.bfloat16, device="cuda").as_strided((n, 1, 128), (pitch, 128, 1)) for _ in range(4)]
    for w, x in zip(wide, (q, k, v)):
        w.copy_(x.cuda())
    out = fp8rl.fp8rl_attention_prompt_bf16(*wide[:3], i32([0, n]), SM, out=wide[3])
    torch.cuda.synchronize()
    check(out, attention.prompt(u16(q), u16(k), u16(v), [0, n], SM), n, attention.BF16_VALUES, "prompt")


def test_prompt_bad_offsets_stay_inside(fp8rl):
    """Offsets outside [0, T] are clamped: no row outside the tensors is touched (the outputs are not specified)."""
    announce("prompt: offsets outside the rows")
    rng = np.random.default_rng(15)
    q, k, v = (bf16(rng, (20, 2, 128)) for _ in range(3))
    out = run_prompt(fp8rl, q, k, v, np.array([-5, 7, 400], np.int32))
    res = attention.prompt(u16(q), u16(k), u16(v), [0, 7, 20], SM)
    check(out, res, 20, attention.BF16_VALUES, "clamped offsets")


def test_prompt_empty_calls(fp8rl):
    announce("prompt: no tokens, no sequences")
    z = torch.empty((0, 2, 128), dtype=torch.bfloat16)
    assert run_prompt(fp8rl, z, z, z, [0, 0]).shape == (0, 2, 128)
    q = torch.ones((3, 2, 128), dtype=torch.bfloat16)
    out = torch.full((3, 2, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    run_prompt(fp8rl, q, q, q, [0], out=out)
    assert torch.all(out == 5.0)


# --------------------------------------------------------------------------
# against the cache
# --------------------------------------------------------------------------
def run_paged(fp8rl, q, kc, vc, table, lens, cu, max_len, sm=0.02, ks=0.02, vs=0.03, out=None, poison=True):
    need = fp8rl.fp8rl_attention_prompt_workspace_size(len(lens), q.shape[0], q.shape[1], kc.shape[1], max_len)
    ws = torch.full((max(need, 16) // 4,), float("nan"), dtype=torch.float32, device="cuda") if poison else None
    out = fp8rl.fp8rl_attention_prompt_fp8kv(
        q.cuda(), torch.from_numpy(kc).cuda(), torch.from_numpy(vc).cuda(), i32(table), i32(lens), i32(cu), max_len,
        f32_1(ks), f32_1(vs), sm, out=out, workspace=ws)
    torch.cuda.synchronize()
    return out


def paged_res(q, kc, vc, table, lens, cu, sm=0.02, ks=np.float32(0.02), vs=np.float32(0.03)):
    return attention.prompt_paged(u16(q), kc, vc, ks, vs, table, lens, cu, sm)


@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (6, 3), (8, 2), (16, 2)])
@pytest.mark.parametrize("lens,new", [([1], [1]), ([0, 5, 16, 0], [0, 5, 16, 2]), ([17, 33, 64], [1, 33, 2]),
                                      ([65, 130, 6], [65, 3, 9]), ([300, 257, 40], [37, 1, 40]), ([700], [60])])
def test_chunk_lengths_and_heads(fp8rl, heads, kv_heads, lens, new):
    """Whole prompts, chunks, single tokens; more new tokens than the sequence has (rows in front of it give 0)."""
    announce(f"chunk {heads}/{kv_heads} heads, lengths {lens}, new {new}")
    rng = np.random.default_rng(heads * 10 + len(lens))
    kc, vc, table = paged(rng, lens, kv_heads, extra_pages=2)
    cu = offsets(new)
    q = bf16(rng, (sum(new), heads, 128))
    out = run_paged(fp8rl, q, kc, vc, table, lens, cu, max(lens) + 20)
    check(out, paged_res(q, kc, vc, table, lens, cu), max(lens), attention.FP8_VALUES, "chunk")
    for b, (n, m) in enumerate(zip(lens, new)):
        if m > n:
            assert torch.all(out[cu[b]:cu[b] + m - n] == 0)
    same(out, run_paged(fp8rl, q, kc, vc, table, lens, cu, max(lens) + 20, poison=False), "not deterministic")


def test_chunk_long_contexts_are_split(fp8rl):
    """Few rows over long sequences of very different lengths, several records each; rows of no sequence stay."""
    announce("chunk: 3 sequences of up to 9001 tokens")
    rng = np.random.default_rng(20)
    lens, new = [9001, 30, 4096], [3, 2, 1]
    assert fp8rl.fp8rl_attention_prompt_workspace_size(3, 10, 4, 1, 9001) > 0, "the case is meant to be split"
    kc, vc, table = paged(rng, lens, 1)
    cu = offsets(new, 1)
    q = bf16(rng, (10, 4, 128))
    q[0], q[7:] = float("nan"), float("nan")
    out = torch.full((10, 4, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    run_paged(fp8rl, q, kc, vc, table, lens, cu, 9001, out=out)
    check(out, paged_res(q, kc, vc, table, lens, cu), 9001, attention.FP8_VALUES, "split chunk")
    assert torch.all(out[0] == 3.0) and torch.all(out[7:] == 3.0)


def test_chunks_give_what_the_whole_prompt_gives(fp8rl):
    """A prompt against the cache at once and in three chunks: the rows differ by no more than both bounds."""
    announce("chunk: a prompt whole and in three chunks")
    rng = np.random.default_rng(21)
    n = 333
    kc, vc, table = paged(rng, [n], 2)
    q = bf16(rng, (n, 4, 128))
    whole = run_paged(fp8rl, q, kc, vc, table, [n], [0, n], n)
    res = paged_res(q, kc, vc, table, [n], [0, n])
    check(whole, res, n, attention.FP8_VALUES, "whole")
    for a, b in ((0, 100), (100, 101), (101, n)):
        part = run_paged(fp8rl, q[a:b], kc, vc, table, [b], [0, b - a], n)
        check(part, [r[a:b] for r in res], n, attention.FP8_VALUES, f"tokens {a} .. {b}")


def test_chunk_tokens_past_max_seq_len_are_ignored(fp8rl):
    announce("chunk: a length above max_seq_len")
    rng = np.random.default_rng(22)
    kc, vc, table = paged(rng, [200], 1)
    q = bf16(rng, (4, 2, 128))
    out = run_paged(fp8rl, q, kc, vc, table, [200], [0, 4], 150)
    check(out, paged_res(q, kc, vc, table, [150], [0, 4]), 150, attention.FP8_VALUES, "chunk")


def test_captured_and_replayed_between_eager_calls(fp8rl):
    """Both entry points in a graph, replayed with new inputs and eager calls between, on a stream of their own."""
    announce("prompt and chunk under a captured graph")
    rng = np.random.default_rng(23)
    lens, new = [2000, 70], [2, 70]
    kc, vc, table = paged(rng, lens, 2)
    cu = offsets(new)
    q, k, v = bf16(rng, (72, 4, 128)).cuda(), bf16(rng, (72, 2, 128)).cuda(), bf16(rng, (72, 2, 128)).cuda()
    args = [torch.from_numpy(kc).cuda(), torch.from_numpy(vc).cuda(), i32(table), i32(lens), i32(cu), 2000, f32_1(0.02),
            f32_1(0.03), 0.02]
    ws = torch.empty(fp8rl.fp8rl_attention_prompt_workspace_size(2, 72, 4, 2, 2000), dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(q), torch.empty_like(q)]

    def both(out):
        fp8rl.fp8rl_attention_prompt_bf16(q, k, v, args[4], SM, out=out[0])
        fp8rl.fp8rl_attention_prompt_fp8kv(q, *args, out=out[1], workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both(outs)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(outs)
    for i in range(4):
        q.copy_(bf16(rng, (72, 4, 128)))
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        want = [torch.empty_like(q), torch.empty_like(q)]
        both(want)
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            same(g, w, f"replay {i}")
