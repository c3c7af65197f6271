"""Chunk appends of many sequences whose caches could take long chunks."""
import numpy as np
import pytest
import torch

from paper_2508_08256_amd import binding as B
from prompt_util import D, starts_of
from test_gpu_prompt_cache import i32, randn

pytestmark = pytest.mark.gpu


def test_more_workgroups_than_one_dimension_of_a_grid_holds():
    """1024 sequences of 8 heads, room for 131072 tokens each, a few hundred tokens and a bound as wide as the arrays: 17.8 million
    workgroups, 4.6e9 threads.  The rows, the codes and the scales are those of the same tokens in a small cache."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    nb, hkv, n, g = 1024, 8, 1 << 17, 256
    rng = np.random.default_rng(1)
    new = rng.integers(0, 2, nb) * rng.integers(1, 200, nb)
    new[-1] = 200
    total = int(new.sum())
    x = torch.zeros(n, 2 * hkv, D, dtype=torch.float16, device="cuda")
    x[:total] = randn((total, 2 * hkv, D), B.F16, 2).cuda()
    starts, lens = i32(starts_of(new)), i32([0] * nb)
    big = B.make_config(nb, hkv, hkv, n, B.F16, group_size=g)
    pools = [torch.zeros(nb, hkv, g, D, dtype=torch.float16, device="cuda") for _ in range(2)]
    table = torch.zeros(nb, n // g, dtype=torch.int32, device="cuda")
    table[:, 0] = torch.arange(nb)
    cache = B.DeviceCache(big, *pools, lens, table)
    B.append_chunk(big, cache, x[:, :hkv], x[:, hkv:], starts, n)
    small = B.make_config(nb, hkv, hkv, g, B.F16, group_size=g)
    flat = [torch.zeros(nb * hkv, g, D, dtype=torch.float16, device="cuda") for _ in range(2)]
    want = B.DeviceCache(small, *flat, lens)
    B.append_chunk(small, want, x[:, :hkv], x[:, hkv:], starts, 200)
    torch.cuda.synchronize()
    assert int(want.k.count_nonzero()) > 0
    assert torch.equal(cache.k.view(-1), want.k.view(-1)) and torch.equal(cache.v.view(-1), want.v.view(-1))
    assert torch.equal(cache.kbits.view(nb * hkv, n * 4)[:, : g * 4], want.kbits.view(nb * hkv, g * 4))
    assert torch.equal(cache.kmeta.view(nb * hkv, -1)[:, :D], want.kmeta.view(nb * hkv, D))
    assert torch.equal(cache.kabsmax, want.kabsmax)
