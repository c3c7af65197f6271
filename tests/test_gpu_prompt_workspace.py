"""One workspace for the attention of chunks and the decode step, as a server would keep it."""
import pytest
import torch

from paper_2508_08256_amd import binding as B
from prompt_util import D, starts_of, tdtype
from test_gpu_prompt_attn import check_chunk, i32, make_cache, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("dtype,block_tokens,n_kv", [(B.BF16, 64, 2), (B.F16, 0, 8)])
def test_chunks_and_decode_steps_share_a_workspace(dtype, block_tokens, n_kv):
    """Side-by-side and shared tiles in many parts, decode steps and dense attention in turn, eagerly and as two captured
    graphs replayed in turn: always what each gives with a workspace of its own."""
    nb, hq, cap, budget = 3, 8, 8192, 300
    cfg = B.make_config(nb, hq, n_kv, cap, dtype)
    first, new = [8000, 2500, 0], [150, 3, 70]
    rows, cache = make_cache(cfg, first, new, dtype, block_tokens, 300)
    for t in (cache.k, cache.v):
        t.nan_to_num_(0.0)  # the decode step appends behind the lengths
    q = randn((sum(new), hq, D), dtype, 301)
    qd, starts = q.cuda(), i32(starts_of(new))
    few, few_starts = q[:6].cuda(), i32([0, 3, 5, 6])
    one = [randn((1, nb, h, D), dtype, 302 + i).cuda() for i, h in enumerate((hq, n_kv, n_kv))]
    budgets = i32([budget] * nb)
    # the decode step works on a copy: it writes rows
    step = B.DeviceCache(cfg, cache.k.clone(), cache.v.clone(), i32([max(f, 1) for f in first]), cache.block_table)
    B.quantize_keys(cfg, step)
    need = max(B.chunk_workspace_bytes(cfg, sum(new), max(new)), B.workspace_bytes(cfg, budget),
               B.workspace_bytes(cfg, cap))
    shared = torch.zeros(need, dtype=torch.uint8, device="cuda")
    own = [torch.zeros(need, dtype=torch.uint8, device="cuda") for _ in range(4)]

    def outputs():
        o16 = dict(dtype=tdtype(dtype), device="cuda")
        return [torch.zeros(sum(new), hq, D, **o16), torch.zeros(6, hq, D, **o16),
                torch.zeros(1, nb, hq, D, device="cuda"), torch.zeros(nb, hq, D, device="cuda")]

    calls = [lambda o, w: B.chunk_attn(cfg, cache, qd, starts, max(new), o, w),
             lambda o, w: B.chunk_attn(cfg, cache, few, few_starts, 3, o, w),
             lambda o, w: B.decode_step(cfg, [step], *one, budgets, budget, o, None, None, w),
             lambda o, w: B.dense_attn(cfg, cache, one[0][0], 0, o, w)]
    want, got = outputs(), outputs()
    for call, o, w in zip(calls, want, own):
        call(o, w)
    torch.cuda.synchronize()
    check_chunk(want[0].cpu(), q, rows, first, new, cfg)

    def check(what):
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(got, want)):
            if i < 2:
                assert torch.equal(a, b), (what, i)
            else:
                # The selection is exact; sums of at most 64 parts may come in another order: each addition is off by 2^-24 of
                # what has been summed, which after the division is at most the largest |v|, in either order.
                assert float((a - b).abs().max()) <= 2 * 64 * 2.0**-24 * float(step.v.abs().max()), (what, i)
            a.zero_()

    for turn in range(3):
        for call, o in zip(calls, got):
            call(o, shared)
        check(("eager", turn))
    graphs = []
    for order in ((0, 2), (3, 1)):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            for i in order:
                calls[i](got[i], shared)
    for turn in range(4):
        for g in graphs if turn % 2 else graphs[::-1]:
            g.replay()
        check(("graphs", turn))
        calls[turn](got[turn], shared)  # eager work in between
        torch.cuda.synchronize()
        got[turn].zero_()
