"""The sum of a row's weights over many tiles of keys: it keeps step with the sum of its values, and neither depends on
the rows beside it."""
import numpy as np
import pytest
import torch

from tests.attn_util import bf16, f32_1, i32, paged, same
from tests.gpu_util import announce, need_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fp8rl():
    need_gpu()
    import paper_2601_18150_amd as m
    m.load()
    return m


def check_ones(out, what):
    """Equal scores weigh equal values of 1: 1, exactly.  The weights are one number, a power of two times 1 + 2^-12 at
    most (the exponent's rounding, half an ulp below 4096), and its rounding to bf16 or fp16 takes no more away; both
    sums and the factor add fp32 roundings, 2 * 8192 of 2^-24 at most: together below 2^-9, half of the step under 1."""
    assert torch.all(out.float() == 1.0), f"{what}: {out.float().min().item()} .. {out.float().max().item()}"


def queries_of(score):
    """(query value, factor): their product with a key of 1.375 is `score`, about, and its product with log2(e) one that
    fp32 rounds up, or down, by as much as any such value's."""
    f = np.float32
    values = np.arange(129, 256) / 128
    factors = [f(abs(score) / (q * 1.375)) for q in values]
    c = [f(s * f(1.4426950408889634)) for s in factors]
    off = [float(f(f(q * 1.375) * x)) - q * 1.375 * float(x) for q, x in zip(values, c)]
    return [(float(np.sign(score) * values[i]), float(factors[i])) for i in (np.argmax(off), np.argmin(off))]


SCORES = [-2700.0, -1400.0, -345.0, 345.0, 1400.0, 2000.0, 2700.0]


@pytest.mark.parametrize("score", SCORES)
def test_many_equal_keys_of_a_prompt(fp8rl, score):
    announce(f"prompt: 8191 tokens of one score, {score}")
    n = 8191
    for query, factor in queries_of(score):
        for heads in (1, 9):                              # tiles of 64 rows, of 128
            q, k, v = (torch.zeros((n, heads, 128), dtype=torch.bfloat16, device="cuda") for _ in range(3))
            q[..., 0], k[..., 0], v[:] = query, 1.375, 1.0
            out = fp8rl.fp8rl_attention_prompt_bf16(q, k, v, i32([0, n]), factor)
            torch.cuda.synchronize()
            check_ones(out, f"{heads} heads, {query} * {factor}")


# (many kv heads or tokens, so that no call divides its keys)
@pytest.mark.parametrize("score", SCORES)
@pytest.mark.parametrize("kv_heads,new", [(520, 2), (16, 2000)])
def test_many_equal_keys_of_a_chunk_and_a_group(fp8rl, score, kv_heads, new):
    announce(f"chunk and shared: {new} tokens, {kv_heads} kv heads, 8000 keys of one score, {score}")
    n = 8000
    kc = torch.zeros((n // 16, kv_heads, 16, 128), dtype=torch.uint8, device="cuda")
    kc[..., 0] = 0x3B                                     # 1.375
    vc = torch.full((n // 16, kv_heads, 4, 128, 4), 0x38, dtype=torch.uint8, device="cuda")   # 1
    one, m = f32_1(1.0), min(new, 100)
    table = torch.arange(n // 16, dtype=torch.int32, device="cuda")[None]
    for query, factor in queries_of(score):
        q = torch.zeros((new, kv_heads, 128), dtype=torch.bfloat16, device="cuda")
        q[..., 0] = query
        out = fp8rl.fp8rl_attention_prompt_fp8kv(q, kc, vc, table, i32([n]), i32([0, new]), n, one, one, factor)
        torch.cuda.synchronize()
        check_ones(out, f"chunk, {query} * {factor}")
        for prefix in (0, 7984):
            out = fp8rl.fp8rl_attention_decode_shared_fp8kv(
                q[:m].contiguous(), kc, vc, table.expand(m, -1).contiguous(), i32([n] * m), i32([0, m]), i32([prefix]), prefix,
                n, one, one, factor)
            torch.cuda.synchronize()
            check_ones(out, f"shared, prefix of {prefix}, {query} * {factor}")


@pytest.mark.parametrize("heads,new,length", [(4, 5, 300), (8, 40, 300), (4, 2, 3000)])
def test_rows_do_not_depend_on_each_other(fp8rl, heads, new, length):
    """The rows beside row 1's head 1 are the same, bit for bit, whatever its scores and whenever its maximum grows."""
    announce(f"chunk, shared and prompt: {new} rows of {heads} heads beside one of other scores")
    rng = np.random.default_rng(new)
    kc, vc, table = paged(rng, [length], 1)
    kc, vc, table, scale = torch.from_numpy(kc).cuda(), torch.from_numpy(vc).cuda(), i32(table), f32_1(0.02)
    n = 400
    q, k, v = bf16(rng, (n, heads, 128), 3.0), bf16(rng, (n, 1, 128), 3.0).cuda(), bf16(rng, (n, 1, 128)).cuda()
    first = None
    for factor in (1.0, -1.0, 20.0, 0.0):
        x = q.clone()
        x[1, 1] = (x[1, 1].float() * factor).to(torch.bfloat16)
        x = x.cuda()
        got = [fp8rl.fp8rl_attention_prompt_fp8kv(x[:new], kc, vc, table, i32([length]), i32([0, new]), length, scale, scale, 0.2),
               fp8rl.fp8rl_attention_decode_shared_fp8kv(x[:new].contiguous(), kc, vc, table.expand(new, -1).contiguous(),
                                                         i32([length] * new), i32([0, new]), i32([160]), 160, length, scale, scale, 0.2),
               fp8rl.fp8rl_attention_prompt_bf16(x, k, v, i32([0, n]), 0.2)]
        torch.cuda.synchronize()
        for g in got:
            g[1, 1] = 0.0
        first = first or got
        for g, f, what in zip(got, first, ("chunk", "shared", "prompt")):
            same(g, f, f"{what}: rows beside one times {factor}")
