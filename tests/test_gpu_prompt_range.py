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


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("first,new,edge", [(30, 8, 32), (100, 200, 128)])
def test_rows_without_a_token_so_far_do_not_round_the_logits_of_others(dtype, first, new, edge):
    """Scaled logits just below 2^22, (2^22 + 0..3) * 0.6 * log2(e) = 3.6e6 and exact before the scale: unrounded they give weights
    within 1e-5, rounded by themselves (the form for larger ones) within 8 % only.  Of the tokens from `edge` on, whose
    wavefront begins there, the first rows see none.  Column d + 4 (token past the edge) of v is 1 for the tokens of logit d: outputs
    are sums of weights of one sign, off by their roundings (u each of the weights and the output, half a step) and those 1e-5."""
    rows = first + new
    cap = -(-rows // 64) * 64
    cfg = B.make_config(1, 1, 1, cap, dtype, sm_scale=0.6)
    j = torch.arange(rows)
    q, k, v = (torch.zeros(n, 1, D, dtype=torch.float64) for n in (new, rows, rows))
    q[:, 0, 0], q[:, 0, 1] = 2048, 1
    k[:, 0, 0], k[:, 0, 1] = 2048, (j % 4).double()
    v[j, 0, j % 4 + 4 * (j >= edge)] = 1
    q, k, v = (t.to(torch.float16 if dtype == F16 else torch.bfloat16) for t in (q, k, v))
    dev = [torch.zeros(1, cap, D, dtype=q.dtype, device="cuda") for _ in range(2)]
    for d, s in zip(dev, (k, v)):
        d[0, :rows] = s[:, 0].cuda()
    out = run_chunk(cfg, B.DeviceCache(cfg, *dev, i32([first])), q, [new])[:, 0].double()
    seen = j[None, :] <= first + torch.arange(new)[:, None]
    want = torch.softmax(torch.where(seen, cfg.sm_scale * (j % 4).double(), -math.inf), dim=1) @ v[:, 0].double()
    u = torch.finfo(q.dtype).eps / 2
    assert bool(((out - want).abs() <= (2 * u + u * u + 1e-5) * want).all()), float(((out - want) / want.clamp(min=1e-9)).abs().max())


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("first,new", [(None, 20), (None, 200), (0, 200), (3000, 3)])
def test_values_that_are_not_finite_show(dtype, bad, first, new):
    """They may not be passed; if one is, the outputs of the rows that attend over it say so."""
    rows = new + (first or 0)
    cap = -(-rows // 64) * 64
    cfg = B.make_config(1, 1, 1, cap, dtype)
    q, k, v = (torch.ones(n, 1, D, dtype=torch.float16 if dtype == F16 else torch.bfloat16) for n in (new, rows, rows))
    v[rows - 2, 0, 5] = bad
    if first is None:
        out = run_prefill(cfg, q, k, v, [new])
    else:
        dev = [torch.zeros(1, cap, D, dtype=q.dtype, device="cuda") for _ in range(2)]
        for d, s in zip(dev, (k, v)):
            d[0, :rows] = s[:, 0].cuda()
        out = run_chunk(cfg, B.DeviceCache(cfg, *dev, i32([first])), q, [new])
    seen = out[new - 2:, 0, 5].float()
    assert not bool(seen.isfinite().any())
    assert bool((out[:, 0, :5] == 1).all())  # equal weights, exact sums: the mean of ones
