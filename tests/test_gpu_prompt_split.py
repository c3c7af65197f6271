"""How the rows of shared tiles are cut: around the numbers of tiles where the rule changes."""
import pytest
import torch

from paper_2508_08256_amd import binding as B
from prompt_util import D, attention64, check_attention
from test_gpu_prompt_attn import make_cache, randn, run_chunk

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("share", [0.45, 0.5, 0.55, 1.15, 1.25, 2.1])
def test_tiles_over_the_places_of_the_gpu(share):
    """128 kv heads of one query head have 6 places each for tiles of 128 tokens.  Every row of three heads against the formula."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    heads, first, new = 128, 700, int(share * 6 * 128) - 3
    cfg = B.make_config(1, heads, heads, 2560, B.BF16)
    rows, cache = make_cache(cfg, [first], [new], B.BF16, 64, 7)
    q = randn((new, heads, D), B.BF16, 8)
    ws = B.make_chunk_workspace(cfg, new, new)
    out = [run_chunk(cfg, cache, q, [new], ws=ws) for _ in range(2)]
    assert torch.equal(*out)
    k, v = (t[0].transpose(0, 1) for t in rows)
    for h in (0, 5, heads - 1):
        want, tol = attention64(q[:, h:h + 1], k[:, h:h + 1], v[:, h:h + 1], first, cfg.sm_scale)
        check_attention(out[0][:, h:h + 1], want, tol, f"head {h}")
