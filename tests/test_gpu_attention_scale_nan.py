"""A key scale that is NaN shows in every row that sees a key, as it does in decode attention, and in no other."""
import numpy as np
import pytest
import torch

from tests.attn_util import bf16, f32_1, i32, offsets, paged
from tests.gpu_util import announce, need_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fp8rl():
    need_gpu()
    import paper_2601_18150_amd as m
    m.load()
    return m


# small tiles and large ones, whole and in records; a row in front of the first token
@pytest.mark.parametrize("heads,lens,new", [(2, [150, 40], [20, 41]), (8, [150, 170], [40, 3]), (4, [2900, 700], [6, 20])])
def test_a_key_scale_of_nan(fp8rl, heads, lens, new):
    announce(f"chunk and shared: {heads} heads, lengths {lens}, new {new}, key scale NaN")
    rng = np.random.default_rng(new[0])
    kc, vc, table = paged(rng, lens, 1)
    kc, vc, cu = torch.from_numpy(kc).cuda(), torch.from_numpy(vc).cuda(), offsets(new)
    q = bf16(rng, (sum(new), heads, 128)).cuda()
    nan, one = f32_1(float("nan")), f32_1(1.0)
    out = fp8rl.fp8rl_attention_prompt_fp8kv(q, kc, vc, i32(table), i32(lens), i32(cu), max(lens), nan, one, 0.1)
    torch.cuda.synchronize()
    for b, (n, m) in enumerate(zip(lens, new)):
        rows = out[int(cu[b]):int(cu[b + 1])]
        none = max(0, m - n)
        assert torch.all(rows[:none] == 0) and torch.isnan(rows[none:]).all()
    for prefix in (0, 32):
        out = fp8rl.fp8rl_attention_decode_shared_fp8kv(q[:2].contiguous(), kc, vc, i32(table), i32(lens), i32([0, 2]), i32([prefix]),
                                                        prefix, max(lens), nan, one, 0.1)
        torch.cuda.synchronize()
        assert torch.isnan(out).all()
    old = fp8rl.fp8rl_attention_decode_fp8kv(q[:2].contiguous(), kc, vc, i32(table), i32(lens), max(lens), nan, one, 0.1)
    torch.cuda.synchronize()
    assert torch.isnan(old).all()
