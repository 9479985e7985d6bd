"""Inputs and checks shared by the attention and page tests (not collected as tests)."""
import numpy as np
import torch

from tests.gpu_util import u16


def bf16(rng, shape, std=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).to(torch.bfloat16)


def offsets(lengths, first=0):
    return np.concatenate([[first], first + np.cumsum(lengths)]).astype(np.int32)


def i32(values):
    return torch.from_numpy(np.ascontiguousarray(values, np.int32)).cuda()


def f32_1(value):
    return torch.tensor([value], dtype=torch.float32, device="cuda")


def codes(rng, shape):
    """Any E4M3 codes but NaN."""
    c = rng.integers(0, 256, shape).astype(np.uint8)
    c[(c & 0x7F) == 0x7F] ^= 1
    return c


def paged(rng, lens, kv_heads, spare=3, extra_pages=0):
    """Caches and a block table for sequences of `lens` tokens over shuffled blocks; NaN codes behind a sequence's end
    and in the blocks of no sequence, ids outside the cache in the entries of no block."""
    pages = [(int(n) + 15) // 16 for n in lens]
    blocks = sum(pages) + spare
    perm = rng.permutation(blocks)
    table = np.where(rng.integers(0, 2, (len(lens), max(max(pages), 1) + extra_pages)) > 0, -7, blocks + 5).astype(np.int32)
    kc, vc = np.full((blocks, kv_heads, 16, 128), 0x7F, np.uint8), np.full((blocks, kv_heads, 4, 128, 4), 0xFF, np.uint8)
    at = 0
    for b, (n, p) in enumerate(zip(lens, pages)):
        table[b, :p] = perm[at:at + p]
        at += p
        for i in range(p):
            t = min(16, int(n) - 16 * i)
            blk = table[b, i]
            kc[blk, :, :t] = codes(rng, (kv_heads, t, 128))
            v = codes(rng, (kv_heads, t, 128))
            for o in range(t):
                vc[blk, :, o // 4, :, o % 4] = v[:, o]
    return kc, vc, table


def check(got: torch.Tensor, res, keys, kind, what):
    """|got - res| within oracle.attention.bound on every element of the rows that belong to a sequence."""
    from oracle import attention
    g = got.float().cpu().numpy().astype(np.float64).reshape(res[0].shape)
    rows = ~np.isnan(res[0])
    err, limit = np.abs(g - res[0]), attention.bound(res, keys, *kind)
    bad = rows & ~(err <= limit)
    assert not bad.any(), (f"{what}: {bad.sum()} of {rows.sum()} outside the bound, first at {tuple(np.argwhere(bad)[0])}: "
                           f"got {g[bad][0]!r}, {res[0][bad][0]!r} +- {limit[bad][0]:.3g}")


def same(a: torch.Tensor, b: torch.Tensor, what):
    assert np.array_equal(u16(a), u16(b)), what
