"""Prompt, chunk and shared attention where scores lie far from zero: single winners and ties of any magnitude, small
differences of large scores, rows beside such rows."""
import numpy as np
import pytest
import torch

from oracle import attention
from tests.attn_util import bf16, check, f32_1, i32, offsets, paged, same
from tests.gpu_util import announce, need_gpu, u16

pytestmark = pytest.mark.gpu
FP8, BF16 = attention.FP8_VALUES, attention.BF16_VALUES
LOG2E = 1.4426950408889634


@pytest.fixture(scope="module")
def fp8rl():
    need_gpu()
    import paper_2601_18150_amd as m
    m.load()
    return m


def chunk(fp8rl, q, kc, vc, table, lens, cu, ks, vs, sm):
    return fp8rl.fp8rl_attention_prompt_fp8kv(q.cuda(), torch.from_numpy(kc).cuda(), torch.from_numpy(vc).cuda(), i32(table),
                                              i32(lens), i32(cu), int(max(lens)), f32_1(ks), f32_1(vs), sm)


def shared(fp8rl, q, kc, vc, table, lens, go, prefix, ks, vs, sm):
    return fp8rl.fp8rl_attention_decode_shared_fp8kv(
        q.cuda(), torch.from_numpy(kc).cuda(), torch.from_numpy(vc).cuda(), i32(table), i32(lens), i32(go), i32(prefix),
        int(max(prefix)), int(max(lens)), f32_1(ks), f32_1(vs), sm)


def exact_scores(res):
    """The oracle's result for scores that are exact in fp32 (sums of few products, or of small whole numbers) and
    differ by 16 at most where they weigh anything: what `bound` counts for their rounding is that of 16."""
    return (res[0], res[1], np.full_like(res[2], 16.0), res[3])


def set_keys(kc, table, lens, dim0):
    """Dim 0 of token t of every sequence becomes dim0[t]'s code."""
    for b, n in enumerate(lens):
        for t in range(int(n)):
            kc[table[b, t // 16], :, t % 16, 0] = dim0[t]


def winners(n, sign):
    """Codes by which the tokens 0, 5, 40, 41, 150 and n - 1 tie and every other scores less by a fourteenth."""
    best, rest = (0x7E, 0x7D) if sign > 0 else (0x7D, 0x7E)      # 448, 416
    dim0 = np.full(n, rest, np.uint8)
    dim0[[t for t in (0, 5, 40, 41, 150, n - 1) if t < n]] = best
    return dim0


def one_dim(rng, shape, power, sign, scale):
    """Queries of dim 0 alone, whose scores are 2^power in units of log2 e, about."""
    q = torch.zeros(shape, dtype=torch.bfloat16)
    q[..., 0] = torch.from_numpy(rng.uniform(0.7, 1.4, shape[:-1])) * (sign * 2.0 ** power / (scale * LOG2E * 448))
    return q


POWERS = [16, 24, 28, 29, 30, 31, 33, 60]


# small tiles and large ones, whole and in records
@pytest.mark.parametrize("heads,lens,new", [(2, [150, 43], [20, 5]), (8, [150, 170], [40, 3]), (4, [2900, 700], [6, 20]),
                                            (8, [1500, 2100], [33, 70])])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("power", POWERS)
def test_ties_of_large_scores_in_a_chunk(fp8rl, heads, lens, new, sign, power):
    announce(f"chunk: {heads} heads, lengths {lens}, new {new}, scores {sign} * 2^{power}")
    rng = np.random.default_rng(power + new[0])
    kc, vc, table = paged(rng, lens, 1)
    set_keys(kc, table, lens, winners(max(lens), sign))
    cu, sm, ks, vs = offsets(new), 0.02, np.float32(0.02), np.float32(0.03)
    q = one_dim(rng, (sum(new), heads, 128), power, sign, sm * ks)
    out = chunk(fp8rl, q, kc, vc, table, lens, cu, ks, vs, sm)
    torch.cuda.synchronize()
    res = attention.prompt_paged(u16(q), kc, vc, ks, vs, table, lens, cu, sm)
    check(out, exact_scores(res), max(lens), FP8, "chunk")


@pytest.mark.parametrize("heads,members", [(2, 3), (8, 40)])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("power", POWERS)
def test_ties_of_large_scores_in_a_group(fp8rl, heads, members, sign, power):
    announce(f"shared: {members} members of {heads} heads, scores {sign} * 2^{power}")
    rng = np.random.default_rng(power + members)
    lens = [900 + int(x) for x in rng.integers(1, 400, members)]
    kc, vc, table = paged(rng, lens, 1)
    table[:, :56] = table[0, :56]
    dim0 = winners(1300, sign)
    dim0[900] = dim0[0]
    set_keys(kc, table, lens, dim0)
    sm, ks, vs = 0.02, np.float32(0.02), np.float32(0.03)
    q = one_dim(rng, (members, heads, 128), power, sign, sm * ks)
    out = shared(fp8rl, q, kc, vc, table, lens, [0, members], [896], ks, vs, sm)
    torch.cuda.synchronize()
    res = attention.prompt_paged(u16(q), kc, vc, ks, vs, table, lens, np.arange(members + 1), sm)
    check(out, exact_scores(res), max(lens), FP8, "shared")


# (up to 512 workgroups take tiles of 64 rows, more of them ones of 128)
@pytest.mark.parametrize("heads,kv_heads", [(2, 1), (180, 180)])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("power", POWERS)
def test_ties_of_large_scores_in_a_prompt(fp8rl, heads, kv_heads, sign, power):
    announce(f"prompt: {heads}/{kv_heads} heads, scores {sign} * 2^{power}")
    rng = np.random.default_rng(power + heads)
    cu, n, sm = [0, 200, 230], 230, 0.02
    k, v = bf16(rng, (n, kv_heads, 128)), bf16(rng, (n, kv_heads, 128))
    for a, b in ((0, 200), (200, 230)):
        best = winners(b - a, sign) == winners(1, sign)[0]
        k[a:b, :, 0] = torch.from_numpy(np.where(best, 448.0 if sign > 0 else 416.0, 416.0 if sign > 0 else 448.0))[:, None].to(k)
    q = one_dim(rng, (n, heads, 128), power, sign, sm)
    out = fp8rl.fp8rl_attention_prompt_bf16(q.cuda(), k.cuda(), v.cuda(), i32(cu), sm)
    torch.cuda.synchronize()
    check(out, exact_scores(attention.prompt(u16(q), u16(k), u16(v), cu, sm)), n, BF16, "prompt")


def steps(rng, n):
    """Whole numbers that rise from 0 to 15 along n tokens, with some noise: maxima that grow from tile to tile."""
    return np.clip(np.arange(n) * 16 // n - rng.integers(0, 4, n), 0, 15)


# (the raw scores are whole numbers below 2^24: exact.  448 * base lies between 2^14 and 2^21)
@pytest.mark.parametrize("base", [-4096, -512, -64, 64, 512, 4096])
def test_small_differences_of_large_scores(fp8rl, base):
    announce(f"chunk, shared and prompt: scores of 448 * {base} + 0 .. 15")
    rng = np.random.default_rng(base + 5000)
    one = np.float32(1.0)
    code = torch.arange(16).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    for heads, lens, new in ((2, [150, 40], [20, 5]), (8, [300, 170], [40, 3]), (4, [2900, 700], [6, 20]), (8, [1500, 2100], [33, 70])):
        kc, vc, table = paged(rng, lens, 1)
        kc[:, :, :, 0] = 0x7E
        for b, n in enumerate(lens):
            t = np.arange(n)
            kc[table[b, t // 16], 0, t % 16, 1] = code[steps(rng, n)]
        cu = offsets(new)
        q = torch.zeros((sum(new), heads, 128), dtype=torch.bfloat16)
        q[..., 0], q[..., 1] = base, 1.0
        out = chunk(fp8rl, q, kc, vc, table, lens, cu, one, one, 1.0)
        res = attention.prompt_paged(u16(q), kc, vc, one, one, table, lens, cu, 1.0)
        check(out, exact_scores(res), max(lens), FP8, f"chunk {new}")
    lens = [1100, 1000, 930]
    kc, vc, table = paged(rng, lens, 1)
    table[:, :56] = table[0, :56]
    kc[:, :, :, 0] = 0x7E
    for b, n in enumerate(lens):
        t = np.arange(n)
        kc[table[b, t // 16], 0, t % 16, 1] = code[steps(rng, n)]
    q = torch.zeros((3, 4, 128), dtype=torch.bfloat16)
    q[..., 0], q[..., 1] = base, 1.0
    out = shared(fp8rl, q, kc, vc, table, lens, [0, 3], [896], one, one, 1.0)
    check(out, exact_scores(attention.prompt_paged(u16(q), kc, vc, one, one, table, lens, np.arange(4), 1.0)), 1100, FP8, "shared")
    for heads in (1, 180):
        k, v = torch.zeros((300, heads, 128), dtype=torch.bfloat16), bf16(rng, (300, heads, 128))
        k[..., 0], k[..., 1] = 448.0, torch.from_numpy(steps(rng, 300)).to(k)[:, None]
        q = torch.zeros((300, heads, 128), dtype=torch.bfloat16)
        q[..., 0], q[..., 1] = base, 1.0
        out = fp8rl.fp8rl_attention_prompt_bf16(q.cuda(), k.cuda(), v.cuda(), i32([0, 300]), 1.0)
        torch.cuda.synchronize()
        some = [0, heads - 1]
        res = attention.prompt(u16(q[:, some]), u16(k[:, some]), u16(v[:, some]), [0, 300], 1.0)
        check(out[:, some], exact_scores(res), 300, BF16, f"prompt of {heads} heads")


@pytest.mark.parametrize("heads,new,length", [(4, 5, 300), (8, 40, 300), (4, 2, 3000)])
def test_rows_beside_one_of_large_scores(fp8rl, heads, new, length):
    """What a row gives does not depend on the rows of its tile."""
    announce(f"chunk and prompt: {new} rows of {heads} heads, one with scores of 2^40")
    rng = np.random.default_rng(new)
    kc, vc, table = paged(rng, [length], 1)
    cu, one = [0, new], np.float32(0.02)
    q = bf16(rng, (new, heads, 128))
    far = q.clone()
    far[1, 1] = (far[1, 1].float() * 2.0 ** 40).to(torch.bfloat16)
    k, v = bf16(rng, (new, 1, 128)), bf16(rng, (new, 1, 128))
    got = []
    for x in (q, far):
        a = chunk(fp8rl, x, kc, vc, table, [length], cu, one, one, 0.05)
        b = fp8rl.fp8rl_attention_prompt_bf16(x.cuda(), k.cuda(), v.cuda(), i32(cu), 0.05)
        torch.cuda.synchronize()
        assert torch.isfinite(a).all() and torch.isfinite(b).all()
        got.append((a.clone(), b.clone()))
    for a, b in zip(*got):
        a[1, 1], b[1, 1] = 0.0, 0.0
        same(a, b, "rows beside it")
