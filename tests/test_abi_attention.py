"""Prompt attention, shared-prefix decode attention and the pages of the cache refuse what they cannot do: through the
C ABI (every argument, built for the host with sanitizers) and through the Python binding, without a GPU."""
import os
import shutil
import subprocess

import pytest
import torch

import paper_2601_18150_amd as fp8rl

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_validation_under_address_and_ub_sanitizers(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not available")
    exe = tmp_path / "abi_attention_asan"
    build = subprocess.run([gxx, "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
                            "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                            f"-I{os.path.join(ROOT, 'include')}",
                            os.path.join(ROOT, "tests", "host", "abi_attention_asan.cpp"), "-o", str(exe)],
                           capture_output=True, text=True)
    if build.returncode != 0 and "asan" in (build.stderr or "").lower():
        pytest.skip("sanitizer runtime not available: " + build.stderr[-200:])
    assert build.returncode == 0, build.stderr[-2000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:verify_asan_link_order=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=120)
    assert run.returncode == 0, run.stdout[-2000:] + run.stderr[-2000:]
    assert run.stdout.startswith("ok"), run.stdout


def bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def i(*values):
    return torch.tensor(values, dtype=torch.int32)


CACHE = [torch.zeros((6, 2, 16, 128), dtype=torch.uint8), torch.zeros((6, 2, 4, 128, 4), dtype=torch.uint8)]
ONE = torch.ones(1)


def prompt(q=bf(5, 8, 128), k=bf(5, 2, 128), v=bf(5, 2, 128), cu=i(0, 5), **kw):
    return fp8rl.fp8rl_attention_prompt_bf16(q, k, v, cu, 0.1, **kw)


def chunk(q=bf(5, 8, 128), k=CACHE[0], v=CACHE[1], table=torch.zeros((2, 3), dtype=torch.int32), lens=i(5, 9), cu=i(0, 2, 5),
          ks=ONE, vs=ONE, **kw):
    return fp8rl.fp8rl_attention_prompt_fp8kv(q, k, v, table, lens, cu, 48, ks, vs, 0.1, **kw)


def shared(q=bf(2, 8, 128), k=CACHE[0], v=CACHE[1], table=torch.zeros((2, 3), dtype=torch.int32), lens=i(5, 9),
           offsets=i(0, 2), prefixes=i(16), ks=ONE, vs=ONE, **kw):
    return fp8rl.fp8rl_attention_decode_shared_fp8kv(q, k, v, table, lens, offsets, prefixes, 16, 48, ks, vs, 0.1, **kw)


def fork(caches=CACHE, table=torch.zeros((4, 3), dtype=torch.int32), lens=i(5, 9, 0, 0), refs=i(0, 0, 0, 0, 0, 0), parents=i(0),
         children=i(2), new=i(5)):
    return fp8rl.fp8rl_kv_fork_sequences(caches, table, lens, refs, parents, children, new)


def compact(caches=CACHE, table=torch.zeros((4, 3), dtype=torch.int32), lens=i(5, 9, 0, 0), refs=i(0, 0, 0, 0, 0, 0), **kw):
    return fp8rl.fp8rl_kv_compact(caches, table, lens, refs, **kw)


@pytest.mark.parametrize("call", [
    lambda: prompt(q=torch.zeros(5, 8, 128)), lambda: prompt(q=bf(5, 1024)), lambda: prompt(k=torch.zeros(5, 2, 128)),
    lambda: prompt(out=torch.zeros(5, 8, 128)), lambda: chunk(k=CACHE[0].float()), lambda: shared(q=bf(2, 8, 128).float()),
    lambda: shared(v=CACHE[1].view(torch.int8)),
])
def test_types_are_refused(call):
    with pytest.raises(TypeError):
        call()


@pytest.mark.parametrize("call", [
    lambda: prompt(k=bf(4, 2, 128)), lambda: prompt(v=bf(5, 1, 128)), lambda: prompt(k=bf(5, 2, 64), v=bf(5, 2, 64)),
    lambda: prompt(cu=torch.tensor([0, 5])), lambda: prompt(cu=i()), lambda: prompt(cu=i(0, 9, 5, 9)[::2]),
    lambda: prompt(q=bf(8, 5, 128).transpose(0, 1)), lambda: prompt(q=bf(5, 8, 256)[..., ::2]),
    lambda: prompt(k=bf(5, 1, 128).expand(5, 2, 128)), lambda: prompt(out=bf(4, 8, 128)),
    lambda: chunk(k=CACHE[0][:, :, :8]), lambda: chunk(k=CACHE[0][:3].contiguous()), lambda: chunk(lens=i(5)),
    lambda: chunk(cu=i(0, 5)), lambda: chunk(table=torch.zeros(2, 3)), lambda: chunk(ks=torch.ones(2)),
    lambda: chunk(vs=torch.ones(1, dtype=torch.float64)), lambda: chunk(workspace=torch.zeros(100)[::2]),
    lambda: shared(offsets=i(0, 1, 2)), lambda: shared(table=torch.zeros((3, 3), dtype=torch.int32)),
    lambda: shared(prefixes=torch.tensor([16])), lambda: shared(out=bf(2, 8, 64)), lambda: shared(lens=i(1, 2, 3)),
    lambda: fork(caches=[]), lambda: fork(caches=[CACHE[0], CACHE[1][:5]]), lambda: fork(caches=[CACHE[0].transpose(0, 1)]),
    lambda: fork(refs=i(0, 0)), lambda: fork(children=i(2, 3)), lambda: fork(lens=i(5)), lambda: fork(new=torch.tensor([5])),
    lambda: compact(live=i(0, 0)), lambda: compact(table=torch.zeros((4, 6), dtype=torch.int32)[:, ::2]),
    lambda: fp8rl.fp8rl_kv_copy_blocks(CACHE, i(1, 2), i(3)),
    lambda: fp8rl.fp8rl_kv_free_sequences(torch.zeros((4, 3), dtype=torch.int32), i(5, 9, 0, 0), i(0, 0), torch.tensor([1])),
])
def test_shapes_are_refused(call):
    with pytest.raises(ValueError):
        call()


@pytest.mark.parametrize("call", [
    lambda: prompt(), lambda: chunk(), lambda: shared(), lambda: fork(), lambda: compact(),
    lambda: fp8rl.fp8rl_kv_copy_blocks(CACHE, i(1), i(3)),
    lambda: fp8rl.fp8rl_kv_free_sequences(torch.zeros((4, 3), dtype=torch.int32), i(5, 9, 0, 0), i(0, 0), i(1)),
])
def test_host_tensors_are_refused(call):
    with pytest.raises(ValueError, match="HIP device"):
        call()


def test_workspace_sizes_are_pure_functions():
    size = fp8rl.fp8rl_attention_prompt_workspace_size
    assert size(3, 12, 32, 8, 20000) > 0 and size(3, 12, 32, 8, 20000) == size(3, 12, 32, 8, 20000)
    assert size(40, 20000, 32, 8, 2000) == 0               # enough tiles without a split
    assert size(0, 12, 32, 8, 100) == 0 and size(3, 12, 32, 5, 100) == 0
    shared_size = fp8rl.fp8rl_attention_decode_shared_workspace_size
    assert shared_size(16, 1, 32, 8, 4000, 6000) > 0 and shared_size(16, 0, 32, 8, 4000, 6000) == 0
    assert shared_size(16, 1, 32, 8, 6001, 6000) == 0
    assert fp8rl.fp8rl_kv_compact_workspace_size(1000) >= 12000
