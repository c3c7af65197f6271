"""Attention of new tokens at the ends of the number ranges."""
import math

import pytest
import torch

from paper_2508_08256_amd import binding as B
from prompt_util import D
from test_gpu_prompt_attn import i32, run_chunk, run_prefill

pytestmark = pytest.mark.gpu
F16, BF16 = B.F16, B.BF16


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("first,new,n_q", [(None, 20, 1), (None, 300, 1), (0, 300, 1), (900, 1, 4), (5000, 4, 4), (3000, 150, 1)])
def test_the_mean_of_the_largest_values_is_finite(first, new, n_q):
    """Every v is +-65504, fp16's largest, and so is every output.  Of 32 tokens one has the weight 1 and the others
    (1 + 1.1 * 2^-11) / 2, which rounds up by 2^-11 * 0.9: weights rounded, over their unrounded sum, give 65530, which as fp16 is an
    infinity.  (first: None for prompts; single tokens, drafts and long chunks over a cache are joined from parts in other places.)"""
    rows = new + (first or 0)
    cap = -(-rows // 64) * 64
    cfg = B.make_config(1, n_q, 1, cap, F16, sm_scale=math.log((1 + 1.1 * 2.0**-11) / 2))
    q, k = torch.zeros(new, n_q, D, dtype=torch.float16), torch.zeros(rows, 1, D, dtype=torch.float16)
    q[:, :, 0] = 1
    k[torch.arange(rows) % 32 != 0, :, 0] = 1
    sign = torch.where(torch.arange(D) % 3 == 0, -1.0, 1.0)
    v = (65504.0 * sign).to(torch.float16).expand(rows, 1, D).contiguous()
    if first is None:
        out = run_prefill(cfg, q, k, v, [new])
    else:
        dev = [torch.zeros(1, cap, D, dtype=torch.float16, device="cuda") for _ in range(2)]
        for d, s in zip(dev, (k, v)):
            d[0, :rows] = s[:, 0].cuda()
        out = run_chunk(cfg, B.DeviceCache(cfg, *dev, i32([first])), q, [new])
    # the true output, and 1 + 2^-11 more of it held to the largest; binary32 is off by far less than half a step, 16
    assert torch.equal(out.double(), (65504.0 * sign.double()).expand(new, n_q, D))
