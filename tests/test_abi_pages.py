"""Lists of caches whose blocks differ are refused by every call that moves blocks, without a GPU."""
import pytest
import torch

import paper_2601_18150_amd as fp8rl


def i(*values):
    return torch.tensor(values, dtype=torch.int32)


TABLE, LENS, REFS = torch.zeros((4, 3), dtype=torch.int32), i(5, 9, 0, 0), i(0, 0, 0, 0, 0, 0)


@pytest.mark.parametrize("call", [
    lambda caches: fp8rl.fp8rl_kv_copy_blocks(caches, i(1), i(2)),
    lambda caches: fp8rl.fp8rl_kv_fork_sequences(caches, TABLE, LENS, REFS, i(0), i(2), i(5)),
    lambda caches: fp8rl.fp8rl_kv_compact(caches, TABLE, LENS, REFS),
])
# blocks of twice and of half the size, in as many bytes; last and in the middle of a list
@pytest.mark.parametrize("shapes", [
    [(6, 2, 16, 128), (3, 4, 16, 128)], [(6, 2, 16, 128), (12, 1, 16, 128)], [(6, 2, 4, 128, 4), (3, 2, 4, 128, 8)],
    [(6, 2, 16, 128), (3, 4, 16, 128), (6, 2, 16, 128)], [(6, 2, 16, 128), (24576,)],
])
def test_caches_of_equal_bytes_and_other_blocks_are_refused(call, shapes):
    with pytest.raises(ValueError, match="one block size"):
        call([torch.zeros(s, dtype=torch.uint8) for s in shapes])


def test_caches_of_one_block_size_and_other_shapes_pass_the_check():
    caches = [torch.zeros(s, dtype=torch.uint8) for s in ((6, 2, 16, 128), (6, 2, 4, 128, 4), (6, 4096))]
    with pytest.raises(ValueError, match="HIP device"):    # (the check behind it)
        fp8rl.fp8rl_kv_compact(caches, TABLE, LENS, REFS)
