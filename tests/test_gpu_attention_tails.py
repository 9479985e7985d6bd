"""One key far in front of a long tail: the tail's values count as much as its weights do, against the FP8 cache too."""
import numpy as np
import pytest
import torch

from oracle import attention
from tests.attn_util import check, f32_1, i32
from tests.gpu_util import announce, need_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fp8rl():
    need_gpu()
    import paper_2601_18150_amd as m
    m.load()
    return m


def want(limits, heads, factor):
    """Rows that see the keys 0 .. limit: key 0 scores 18 * factor and has values 0, the others score 0 and have 448."""
    tail = limits * np.exp(-18.0 * float(factor))
    rows = np.broadcast_to((448.0 * tail / (1.0 + tail))[:, None, None], (len(limits), heads, 128))
    per_head = np.ones((len(limits), heads))
    return rows, rows, 18.0 * float(factor) * per_head, 448.0 * per_head


# the tail's weights, as powers of 2: on both sides of fp16's normal numbers, of what it holds at all, and far below
@pytest.mark.parametrize("power", [-10.0, -13.9, -16.3, -20.7, -24.4, -25.1, -26.0, -28.3, -30.6])
# few rows and many, over keys in one share (many kv heads, or tokens) and in several; all tokens of one length
@pytest.mark.parametrize("kv_heads,group,new,n", [(520, 1, 2, 20000), (16, 1, 2000, 20000), (1, 8, 3, 131072), (1, 8, 40, 70000)])
def test_a_long_tail_behind_one_key(fp8rl, kv_heads, group, new, n, power):
    announce(f"chunk and shared: {new} tokens, {kv_heads} kv heads, {n} keys, tail of 2^{power}")
    factor = np.float32(-power / (18.0 * np.log2(np.e)))
    kc = torch.zeros((n // 16, kv_heads, 16, 128), dtype=torch.uint8, device="cuda")
    kc[0, :, 0, 0] = 0x59                                  # 18
    vc = torch.full((n // 16, kv_heads, 4, 128, 4), 0x7E, dtype=torch.uint8, device="cuda")
    vc[0, :, 0, :, 0] = 0
    q = torch.zeros((new, kv_heads * group, 128), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    one, m = f32_1(1.0), min(new, 100)
    table = torch.arange(n // 16, dtype=torch.int32, device="cuda")[None]
    out = fp8rl.fp8rl_attention_prompt_fp8kv(q, kc, vc, table, i32([n]), i32([0, new]), n, one, one, float(factor))
    torch.cuda.synchronize()
    heads = [0, kv_heads * group - 1]
    check(out[:, heads], want(np.arange(n - new, n), 2, factor), n, attention.FP8_VALUES, "chunk")
    for prefix in (0, n // 16 * 16 - 16):
        out = fp8rl.fp8rl_attention_decode_shared_fp8kv(
            q[:m].contiguous(), kc, vc, table.expand(m, -1).contiguous(), i32([n] * m), i32([0, m]), i32([prefix]), prefix, n,
            one, one, float(factor))
        torch.cuda.synchronize()
        check(out[:, heads], want(np.full(m, n - 1), 2, factor), n, attention.FP8_VALUES, f"shared, prefix of {prefix}")


@pytest.mark.parametrize("power", [-10.0, -25.1, -30.6, -60.0])
@pytest.mark.parametrize("heads", [1, 9])                 # tiles of 64 rows, of 128
def test_a_long_tail_in_a_prompt(fp8rl, heads, power):
    announce(f"prompt: 20000 tokens, {heads} heads, tail of 2^{power}")
    n, factor = 20000, np.float32(-power / (18.0 * np.log2(np.e)))
    q, k = (torch.zeros((n, heads, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q[..., 0], k[0, :, 0] = 1.0, 18.0
    v = torch.full((n, heads, 128), 448.0, dtype=torch.bfloat16, device="cuda")
    v[0] = 0.0
    out = fp8rl.fp8rl_attention_prompt_bf16(q, k, v, i32([0, n]), float(factor))
    torch.cuda.synchronize()
    some = np.array([0, 1, 63, 64, 127, 128, 5000, n - 1])
    check(out[some.tolist()][:, [0]], want(some, 1, factor), n, attention.BF16_VALUES, "prompt")
