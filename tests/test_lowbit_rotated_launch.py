"""How far the launch of rotated cache writes reaches: workgroups for each page, head and four queries, which can be more than an axis of a launch holds (2^32 threads)."""
import ctypes as C

import pytest
import torch

from test_gpu_lowbit_rotated import Both

P = 0x1000                                                 # never dereferenced


@pytest.fixture(scope="module")
def lowbit():
    import os
    from paper_2604_03298_amd import enec, lowbit as module
    if not os.path.exists(enec.LIB_PATH):
        from paper_2604_03298_amd import build
        build.build()
    module.lib()
    return module


def blocks_of(batch, tokens, page, kv, group):
    return (tokens // page + 2 * batch) * kv * (2 + (group + 3) // 4)


@pytest.mark.parametrize("batch, tokens, page, kv, group", [(65535, 5, 64, 65535, 1), (65535, 65535, 16, 8192, 0), (4096, 16, 64, 16, 65535)])
def test_more_workgroups_than_can_be_numbered_are_refused(lowbit, batch, tokens, page, kv, group):
    assert blocks_of(batch, tokens, page, kv, group) >= 1 << 31
    cache = lowbit.CacheStruct(P, P, P, P, 10, page, kv, 64)
    b = lowbit.BatchStruct(P, P, P, 8, batch, tokens, None)
    q, out = (P, 0x2000) if group else (None, None)
    assert lowbit.lib().enec_cache_write_rotated(C.byref(cache), C.byref(b), P, 64, 64, P, 64, 64, q, 64, 64, out, 64, 64, kv * group, 0, P, 100, 64, 0, None) == lowbit.E_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_more_workgroups_than_an_axis_holds(lowbit, interleaved):
    """Workgroups of 256 threads, more than 2^24 of them; the tokens are those of the first, a middle and the last sequences, one of them idle."""
    batch, group, dim, page = 600, 65535, 64, 256
    new, lengths = [0] * batch, [0] * batch
    new[0], new[300], new[-2], new[-1] = 1, 2, 1, 2
    lengths[0], lengths[300], lengths[-1] = 1, 9, 2
    assert 1 << 24 < blocks_of(batch, sum(new), page, 1, group) < 1 << 31
    both = Both(lowbit, 5, batch, 1, dim, page, 1, 32, 20, interleaved, torch.float16)
    both.write([7 if b == 300 else 0 for b in range(batch)], [7 if b == 300 else 0 for b in range(batch)], 0)
    both.write(new, lengths, group)
    both.check()
