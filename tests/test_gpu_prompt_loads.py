"""Rows loaded with and without the hint for data that is read once."""
import pytest
import torch

from paper_2508_08256_amd import binding as B
from prompt_util import D, attention64, check_attention
from test_gpu_prompt_attn import i32, randn, run_chunk

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,rows", [(8, 65408), (8, 65600), (32, 16320), (32, 16448)])
def test_single_tokens_over_rows_around_the_last_caches_size(heads, rows):
    """256 MiB of K and V, a little less and a little more."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cfg = B.make_config(1, heads, heads, rows, B.BF16)
    k, v = (torch.randn(heads, rows, D, generator=torch.Generator().manual_seed(s)).to(torch.bfloat16) for s in (1, 2))
    cache = B.DeviceCache(cfg, k.cuda(), v.cuda(), i32([rows - 1]))
    q = randn((1, heads, D), B.BF16, 3)
    out = run_chunk(cfg, cache, q, [1])
    want, tol = attention64(q, k.transpose(0, 1), v.transpose(0, 1), rows - 1, cfg.sm_scale)
    check_attention(out, want, tol)
