"""Causal attention of prompts and of chunks of new tokens over a cache, against the formula in 64 bits."""
import math
import os

import numpy as np
import pytest
import torch

from paper_2508_08256_amd import binding as B
from prompt_util import D, attention64, check_attention, starts_of, tdtype

pytestmark = pytest.mark.gpu
F16, BF16 = B.F16, B.BF16


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def i32(a):
    return torch.as_tensor(np.asarray(a, np.int32), device="cuda")


def randn(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(tdtype(dtype))


SENTINEL = 7.0


def run_prefill(cfg, q, k, v, lens, pad=0, max_new=None, fused=False):
    n = q.shape[0]
    fill = lambda t: torch.cat([t, torch.full((pad, *t.shape[1:]), math.nan, dtype=t.dtype)])  # noqa: E731
    qd, kd, vd = fill(q).cuda(), fill(k).cuda(), fill(v).cuda()
    if fused:
        both = torch.cat([qd, kd, vd], dim=1)
        qd, kd, vd = both.split([q.shape[1], k.shape[1], v.shape[1]], dim=1)
    out = torch.full((n + pad, q.shape[1], D), SENTINEL, dtype=q.dtype, device="cuda")
    B.prefill_attn(cfg, qd, kd, vd, i32(starts_of(lens)), max(lens) if max_new is None else max_new, out)
    torch.cuda.synchronize()
    return out.cpu()


def check_prefill(out, q, k, v, lens, scale):
    at = 0
    for b, n in enumerate(lens):
        if n:
            want, tol = attention64(q[at:at + n], k[at:at + n], v[at:at + n], 0, scale)
            check_attention(out[at:at + n], want, tol, f"sequence {b}")
        at += n
    assert bool((out[at:] == SENTINEL).all())


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("n_q,n_kv", [(1, 1), (4, 4), (8, 4), (3, 1), (8, 2), (10, 2), (6, 1), (7, 1), (16, 2)])
def test_prompts_of_unequal_lengths(dtype, n_q, n_kv):
    """Lengths around the tiles of 32 and 64, none, one; every number of heads that share a kv head."""
    lens = [1, 0, 33, 64, 65, 127, 200]
    n = sum(lens)
    cfg = B.make_config(len(lens), n_q, n_kv, 256, dtype)
    q, k, v = randn((n, n_q, D), dtype, 1), randn((n, n_kv, D), dtype, 2), randn((n, n_kv, D), dtype, 3)
    for fused in (False, True):
        check_prefill(run_prefill(cfg, q, k, v, lens, pad=5, fused=fused), q, k, v, lens, cfg.sm_scale)


@pytest.mark.parametrize("dtype,n_q,n_kv,n", [(F16, 2, 2, 1500), (BF16, 4, 1, 1025), (F16, 8, 1, 700), (BF16, 1, 1, 2049), (BF16, 32, 32, 300), (F16, 24, 8, 777)])
def test_long_prompts(dtype, n_q, n_kv, n):
    cfg = B.make_config(1, n_q, n_kv, 4096, dtype)
    q, k, v = randn((n, n_q, D), dtype, 4, 1.5), randn((n, n_kv, D), dtype, 5, 1.5), randn((n, n_kv, D), dtype, 6)
    check_prefill(run_prefill(cfg, q, k, v, [n]), q, k, v, [n], cfg.sm_scale)


def test_offsets_that_make_no_sense_stay_inside_the_arrays():
    """Descending, negative and too large offsets, more tokens than max_new: rows outside are not touched, the first max_new
    tokens of a sequence are right."""
    cfg = B.make_config(4, 2, 1, 128, BF16)
    q, k, v = randn((50, 2, D), BF16, 7), randn((50, 1, D), BF16, 8), randn((50, 1, D), BF16, 9)
    out = torch.full((50, 2, D), SENTINEL, dtype=torch.bfloat16, device="cuda")
    B.prefill_attn(cfg, q.cuda(), k.cuda(), v.cuda(), i32([0, 20, -5, 40, 1 << 30]), 12, out)
    torch.cuda.synchronize()
    out = out.cpu()
    for lo in (0, 40):  # 0..19 cut at 12; 20..-5: none; -5..40 begins at 0, cut; 40..50
        n = min(12, 50 - lo)
        want, tol = attention64(q[lo:lo + n], k[lo:lo + n], v[lo:lo + n], 0, cfg.sm_scale)
        check_attention(out[lo:lo + n], want, tol)
    assert bool((out[12:40] == SENTINEL).all())


@pytest.mark.parametrize("scale", [-0.3, 0.0, 3e4])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_softmax_scales(dtype, scale):
    """A negative scale, zero (the mean of V) and one under which the largest logit takes all the weight."""
    n = 150
    cfg = B.make_config(1, 4, 2, 256, dtype, sm_scale=scale)
    q, k, v = randn((n, 4, D), dtype, 10), randn((n, 2, D), dtype, 11), randn((n, 2, D), dtype, 12)
    if abs(scale) > 1:
        # the two largest logits of a row must differ by more than binary32 can blur
        q, k = q.sign() * torch.ones_like(q), k.sign() * torch.ones_like(k)
        k[torch.arange(n), :, :] = 1
        q[:] = 1
        k[:, :, 0] = torch.arange(n, dtype=torch.float32)[:, None].to(k.dtype) - (torch.arange(n) == 40).to(k.dtype)[:, None] * 40
    got = run_prefill(cfg, q, k, v, [n])
    if abs(scale) > 1:
        best = torch.tensor([i - 1 if i == 40 else i for i in range(n)])
        # One weight p, the others exp2(-4e4) = 0: the result is round(round(p) v / p), each rounding within a factor 1 + u, and
        # p = 1 only up to the rounding of its logit, so round(p) / p need not be 1.
        u = torch.finfo(got.dtype).eps / 2
        for h, kv in ((0, 0), (3, 1)):
            w = v[best, kv].double()
            assert bool(((got[:, h].double() - w).abs() <= (2 * u + u * u + 1e-6) * w.abs() + 2.0**-25).all())
    else:
        check_prefill(got, q, k, v, [n], cfg.sm_scale)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_logits_far_beyond_24_bits(dtype):
    """Equal rows under huge logits: the mean of V.  (Weights must not move with the rounding of the largest logit.)"""
    n, big = 90, (250.0 if dtype == F16 else 1e15)
    cfg = B.make_config(1, 2, 1, 128, dtype, sm_scale=1e3)
    q = torch.full((n, 2, D), big).to(tdtype(dtype))
    k = torch.full((n, 1, D), big).to(tdtype(dtype))
    v = randn((n, 1, D), dtype, 13)
    got = run_prefill(cfg, q, k, v, [n])
    mean = v[:, 0].double().cumsum(0) / torch.arange(1, n + 1)[:, None]
    size = v[:, 0].double().abs().cumsum(0) / torch.arange(1, n + 1)[:, None]
    u = torch.finfo(tdtype(dtype)).eps / 2
    assert bool(((got[:, 0].double() - mean).abs() <= u * mean.abs() + (u + 1e-5) * size + 1e-7).all())


def make_cache(cfg, first, new, dtype, block_tokens, seed):
    """Rows [0, first + new) of every sequence random, everything else NaN; K, V per sequence on the host too."""
    cap, nb, hkv = cfg.max_ctx, cfg.batch, cfg.n_kv_heads
    rows = []
    for which in (0, 1):
        t = torch.full((nb, hkv, cap, D), math.nan, dtype=tdtype(dtype))
        for b in range(nb):
            n = min(cap, first[b] + new[b])
            t[b, :, :n] = randn((hkv, n, D), dtype, seed + 10 * b + which)
        rows.append(t)
    table = None
    dev = [t.view(nb * hkv, cap, D).cuda() for t in rows]
    if block_tokens:
        per = cap // block_tokens
        perm = torch.randperm(nb * per + 3, generator=torch.Generator().manual_seed(seed))
        table = perm[: nb * per].view(nb, per).to(torch.int32)
        pools = []
        for t in rows:
            pool = torch.full((nb * per + 3, hkv, block_tokens, D), math.nan, dtype=t.dtype)
            pool[table.long()] = t.view(nb, hkv, per, block_tokens, D).transpose(1, 2)
            pools.append(pool.cuda())
        dev, table = pools, table.cuda()
    return rows, B.DeviceCache(cfg, dev[0], dev[1], i32(first), table)


def run_chunk(cfg, cache, q, new, pad=0, ws=None, max_new=None):
    qd = torch.cat([q, torch.full((pad, *q.shape[1:]), math.nan, dtype=q.dtype)]).cuda()
    out = torch.full(qd.shape, SENTINEL, dtype=q.dtype, device="cuda")
    max_new = max(max(new), 1) if max_new is None else max_new
    ws = B.make_chunk_workspace(cfg, qd.shape[0], max_new) if ws is None else ws
    B.chunk_attn(cfg, cache, qd, i32(starts_of(new)), max_new, out, ws)
    torch.cuda.synchronize()
    return out.cpu()


def check_chunk(out, q, rows, first, new, cfg):
    at = 0
    for b, n in enumerate(new):
        if n:
            k, v = (t[b].transpose(0, 1) for t in rows)
            want, tol = attention64(q[at:at + n], k, v, first[b], cfg.sm_scale, cap=cfg.max_ctx)
            check_attention(out[at:at + n], want, tol, f"sequence {b}")
        at += n
    assert bool((out[at:] == SENTINEL).all())


@pytest.mark.parametrize("block_tokens", [0, 64, 256])
@pytest.mark.parametrize("dtype,n_q,n_kv", [(F16, 4, 4), (BF16, 8, 2), (BF16, 6, 2), (F16, 8, 1), (BF16, 5, 1), (F16, 14, 2)])
def test_chunks_of_unequal_lengths(dtype, n_q, n_kv, block_tokens):
    first = [0, 63, 64, 500, 1000, 127, 1]
    new = [70, 1, 0, 33, 9, 130, 64]
    cfg = B.make_config(len(first), n_q, n_kv, 1280, dtype)
    rows, cache = make_cache(cfg, first, new, dtype, block_tokens, 20)
    q = randn((sum(new), n_q, D), dtype, 21)
    check_chunk(run_chunk(cfg, cache, q, new, pad=3), q, rows, first, new, cfg)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("n_q,n_kv", [(1, 1), (2, 1), (8, 1), (8, 8), (12, 4)])
@pytest.mark.parametrize("new", [1, 2, 5])
def test_single_and_drafted_tokens_over_long_caches(dtype, n_q, n_kv, new):
    """Few rows: the caches are split over many workgroups.  Lengths from an empty cache to 9000, blocks that end anywhere."""
    first = [0, 31, 2047, 9000]
    cfg = B.make_config(4, n_q, n_kv, 9216, dtype)
    rows, cache = make_cache(cfg, first, [new] * 4, dtype, 64 if new == 2 else 0, 30 + new)
    q = randn((4 * new, n_q, D), dtype, 31)
    ws = B.make_chunk_workspace(cfg, 4 * new, new)
    for _ in range(3):  # the workspace is left ready for the next call
        check_chunk(run_chunk(cfg, cache, q, [new] * 4, ws=ws), q, rows, first, [new] * 4, cfg)


@pytest.mark.parametrize("dtype,n_q,n_kv,first,new", [(BF16, 8, 2, 5000, 300), (F16, 4, 4, 3001, 129), (BF16, 1, 1, 20000, 40), (F16, 16, 2, 700, 600)])
def test_long_chunks_behind_long_contexts(dtype, n_q, n_kv, first, new):
    cap = -(-(first + new) // 64) * 64
    cfg = B.make_config(1, n_q, n_kv, cap, dtype)
    rows, cache = make_cache(cfg, [first], [new], dtype, 64, 40)
    q = randn((new, n_q, D), dtype, 41)
    check_chunk(run_chunk(cfg, cache, q, [new]), q, rows, [first], [new], cfg)


def test_many_tiles_and_parts_of_unequal_numbers():
    """One call with every way a tile's rows are split: 48 parts in groups and fewer, single tokens beside them; then far more tiles
    than there are counters for groups.  The workspace is left ready each time."""
    cfg = B.make_config(5, 8, 1, 16384, BF16)
    first, new = [9000, 16000, 3000, 0, 12000], [150, 4, 17, 900, 1]
    rows, cache = make_cache(cfg, first, new, BF16, 64, 80)
    q = randn((sum(new), 8, D), BF16, 81)
    ws = B.make_chunk_workspace(cfg, sum(new), max(new))
    for _ in range(2):
        check_chunk(run_chunk(cfg, cache, q, new, ws=ws), q, rows, first, new, cfg)
    for n, lo in ((1010, 2000), (8200, 300)):
        cfg = B.make_config(1, 8, 1, 16384, BF16)
        rows, cache = make_cache(cfg, [lo], [n], BF16, 64, 82)
        q = randn((n, 8, D), BF16, 83)
        ws = B.make_chunk_workspace(cfg, n, n)
        out = [run_chunk(cfg, cache, q, [n], ws=ws) for _ in range(2)]
        assert torch.equal(*out)
        k, v = (t[0].transpose(0, 1) for t in rows)
        for at in sorted({0, 1, 500, n - 700, n - 1}):  # single rows of it
            want, tol = attention64(q[at:at + 1], k, v, lo + at, cfg.sm_scale)
            check_attention(out[0][at:at + 1], want, tol, str(at))


def test_a_batch_of_more_sequences_than_lanes():
    """130 sequences, tokens in every third."""
    n = 130
    cfg = B.make_config(n, 4, 2, 640, F16)
    rng = np.random.default_rng(3)
    first = rng.integers(0, 500, n).tolist()
    new = [int(rng.integers(1, 100)) if b % 3 == 0 else (b % 2 if b > 100 else 0) for b in range(n)]
    rows, cache = make_cache(cfg, first, new, F16, 0, 84)
    q = randn((sum(new), 4, D), F16, 85)
    check_chunk(run_chunk(cfg, cache, q, new, pad=2), q, rows, first, new, cfg)


def test_offsets_that_make_no_sense_leave_the_workspace_ready():
    """Sequences that share tokens, more of them than there are tokens: whatever comes out, the next call is right."""
    cfg = B.make_config(6, 2, 1, 4096, BF16)
    first, new = [4000, 3000, 2000, 4000, 10, 500], [10, 0, 40, 1, 30, 2]
    rows, cache = make_cache(cfg, first, new, BF16, 0, 86)
    q = randn((sum(new), 2, D), BF16, 87)
    ws = B.make_chunk_workspace(cfg, sum(new), max(new))
    out = torch.zeros(sum(new), 2, D, dtype=torch.bfloat16, device="cuda")
    for bad in ([0, 83, 0, 83, 0, 83, 0], [83, 0, 1 << 30, -1, 50, 20, 83], [-5, 40, 0, 40, 0, 40, 83]):
        B.chunk_attn(cfg, cache, q.cuda(), i32(bad), 83, out, ws)
    check_chunk(run_chunk(cfg, cache, q, new, ws=ws), q, rows, first, new, cfg)


def test_a_full_cache():
    """Tokens past the capacity attend over all of its rows; lengths above it count as full, below 0 as empty."""
    cfg = B.make_config(3, 4, 2, 256, BF16)
    first, new = [250, 256, 0], [20, 3, 2]
    rows, cache = make_cache(cfg, first, new, BF16, 64, 50)
    cache.seq_lens.copy_(i32([250, 300, -4]))
    q = randn((25, 4, D), BF16, 51)
    check_chunk(run_chunk(cfg, cache, q, new), q, rows, first, new, cfg)


def test_chunks_on_another_stream_and_in_a_graph():
    """Captured with two workspaces in one graph, replayed with eager work on the first in between: the eager result."""
    cfg = B.make_config(2, 8, 2, 4096, BF16)
    first, new = [4000, 1200], [4, 2]
    rows, cache = make_cache(cfg, first, new, BF16, 64, 60)
    q = randn((6, 8, D), BF16, 61)
    want = run_chunk(cfg, cache, q, new)
    check_chunk(want, q, rows, first, new, cfg)
    qd, starts = q.cuda(), i32(starts_of(new))
    ws = [B.make_chunk_workspace(cfg, 6, 4) for _ in range(2)]
    outs = [torch.zeros(6, 8, D, dtype=q.dtype, device="cuda") for _ in range(3)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.chunk_attn(cfg, cache, qd, starts, 4, outs[2], ws[0])
    side.synchronize()
    assert torch.equal(outs[2].cpu(), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for o, w in zip(outs, ws):
            B.chunk_attn(cfg, cache, qd, starts, 4, o, w)
    for _ in range(4):
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0].cpu(), want) and torch.equal(outs[1].cpu(), want)
        B.chunk_attn(cfg, cache, qd, starts, 4, outs[2], ws[0])
        torch.cuda.synchronize()
        assert torch.equal(outs[2].cpu(), want)


def test_results_do_not_change_from_call_to_call():
    cfg = B.make_config(2, 8, 8, 2048, F16)
    rows, cache = make_cache(cfg, [2000, 700], [3, 1], F16, 0, 70)
    q = randn((4, 8, D), F16, 71)
    ws = B.make_chunk_workspace(cfg, 4, 3)
    ref = run_chunk(cfg, cache, q, [3, 1], ws=ws)
    for _ in range(10):
        assert torch.equal(run_chunk(cfg, cache, q, [3, 1], ws=ws), ref)


def test_only_padding():
    """Rows in the arrays, no tokens in any sequence."""
    cfg = B.make_config(3, 4, 2, 256, BF16)
    rows, cache = make_cache(cfg, [0, 5, 256], [0, 0, 0], BF16, 0, 90)
    q = torch.zeros(0, 4, D, dtype=torch.bfloat16)
    assert bool((run_chunk(cfg, cache, q, [0, 0, 0], pad=9, max_new=9) == SENTINEL).all())
    assert bool((run_prefill(cfg, q, q[:, :2], q[:, :2], [0, 0, 0], pad=9, max_new=9) == SENTINEL).all())


RANDOM = range(int(os.environ.get("FIER_RANDOM_PROMPT_SEEDS", "24")))


def random_shape(seed):
    rng = np.random.default_rng(seed)
    hkv = int(rng.choice([1, 2, 3, 5]))
    return rng, int(rng.integers(1, 7)), hkv * int(rng.integers(1, 9)), hkv, int(rng.choice([F16, BF16]))


def edges(rng, most, n):
    """Lengths: around multiples of 32, of 64 and of 96, small ones, anything."""
    kind = rng.integers(0, 4, n)
    near = rng.choice([32, 64, 96, 128], n) * rng.integers(0, 8, n) + rng.integers(-1, 2, n)
    x = np.where(kind == 0, near, np.where(kind == 1, rng.integers(0, 4, n), rng.integers(0, most + 1, n)))
    return np.clip(x, 0, most)


@pytest.mark.parametrize("seed", RANDOM)
def test_random_prompts(seed):
    rng, nb, hq, hkv, dtype = random_shape(seed)
    lens = edges(rng, 500, nb).tolist()
    n = sum(lens)
    cfg = B.make_config(nb, hq, hkv, 512, dtype, sm_scale=float(rng.choice([0.0884, 0.02, -0.05])))
    q, k, v = randn((n, hq, D), dtype, 3 * seed + 1), randn((n, hkv, D), dtype, 3 * seed + 2), randn((n, hkv, D), dtype, 3 * seed + 3)
    out = run_prefill(cfg, q, k, v, lens, pad=int(rng.integers(0, 3)), max_new=max(lens) + int(rng.integers(0, 50)), fused=bool(seed % 2))
    check_prefill(out, q, k, v, lens, cfg.sm_scale)


@pytest.mark.parametrize("seed", RANDOM)
def test_random_chunks(seed):
    rng, nb, hq, hkv, dtype = random_shape(1000 + seed)
    most = int(rng.choice([1, 4, 40, 300]))
    new = edges(rng, most, nb).tolist()
    new[-1] = max(1, new[-1])
    first = edges(rng, int(rng.choice([300, 4000])), nb).tolist()
    g = int(rng.choice([32, 128]))
    bt = int(rng.choice([0, 128, 256]))
    cap = -(-max(f + n for f, n in zip(first, new)) // 256) * 256 + 256 * int(rng.integers(0, 2))
    cfg = B.make_config(nb, hq, hkv, cap, dtype, group_size=g)
    rows, cache = make_cache(cfg, first, new, dtype, bt, 5000 + 50 * seed)
    q = randn((sum(new), hq, D), dtype, 6000 + seed)
    pad = int(rng.integers(0, 3))
    ws = B.make_chunk_workspace(cfg, sum(new) + pad, max(new) + 3)
    for _ in range(2):
        out = run_chunk(cfg, cache, q, new, pad=pad, ws=ws, max_new=max(new) + 3)
        check_chunk(out, q, rows, first, new, cfg)


# ---- addresses beyond 32 bits ------------------------------------------------------------------------------------------------


def attention64_gpu(q, k, v, first, scale):
    """One head, a query row at a time: (outputs, tolerances) as attention64's."""
    o, t = [], []
    u = torch.finfo(q.dtype).eps / 2
    for i in range(q.shape[0]):
        x = q[i].double()
        kk, vv = k[: first + i + 1].double(), v[: first + i + 1].double()
        w = torch.softmax(scale * (kk @ x), dim=0)
        a = float((kk.abs() @ x.abs()).max()) * abs(scale)
        y = w @ vv
        o.append(y)
        t.append((u + 2 * 132 * 2.0**-24 * a + 1e-5) * (w @ vv.abs()) * 1.01 + u * y.abs() + 2.0**-24 + 2.0**-32 * vv.abs().sum(dim=0))
    return torch.stack(o).cpu(), torch.stack(t).cpu()


def test_a_cache_of_more_than_four_gigabytes():
    """Two sequences of 2^20 rows, 8 kv heads: 4.3 GB each of K and V.  Chunks into the last rows, attention over all of them."""
    cfg = B.make_config(2, 8, 8, 1 << 20, BF16)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    k, v = (torch.empty(16, 1 << 20, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t in (k, v):
        for u in range(16):
            t[u] = torch.randn((1 << 20, D), generator=gen, device="cuda")
    first, new = [7, (1 << 20) - 5], [2, 5]
    cache = B.DeviceCache(cfg, k, v, i32(first))
    x = randn((7, 24, D), BF16, 91).cuda()
    starts = i32(starts_of(new))
    B.append_chunk(cfg, cache, x[:, 8:16], x[:, 16:], starts, 5)
    out = torch.zeros(7, 8, D, dtype=torch.bfloat16, device="cuda")
    B.chunk_attn(cfg, cache, x[:, :8], starts, 5, out, B.make_chunk_workspace(cfg, 7, 5))
    torch.cuda.synchronize()
    for h in (0, 7):
        assert torch.equal(k[8 + h, -5:], x[2:, 8 + h]) and torch.equal(v[8 + h, -5:], x[2:, 16 + h])
        assert torch.equal(k[h, 7:9], x[:2, 8 + h])
        for b, at in ((0, 0), (1, 2)):
            want, tol = attention64_gpu(x[at:at + new[b], h], k[8 * b + h], v[8 * b + h], first[b], cfg.sm_scale)
            check_attention(out[at:at + new[b], h], want, tol, f"sequence {b} head {h}")


def test_a_pool_of_more_than_four_gigabytes():
    cfg = B.make_config(1, 8, 8, 1024, F16)
    n_pool = (1 << 32) // (8 * 64 * D * 2) + 40  # blocks of 64 rows of 8 heads
    k, v = (torch.empty(n_pool, 8, 64, D, dtype=torch.float16, device="cuda") for _ in range(2))
    table = torch.arange(n_pool - 16, n_pool, dtype=torch.int32).flip(0).view(1, 16).contiguous()
    for t in (k, v):
        t[table[0].long().cuda()] = float("nan")
    cache = B.DeviceCache(cfg, k, v, i32([0]), table.cuda())
    x = randn((700, 24, D), F16, 92)
    xd, starts = x.cuda(), i32([0, 700])
    B.append_chunk(cfg, cache, xd[:, 8:16], xd[:, 16:], starts, 700)
    out = torch.zeros(700, 8, D, dtype=torch.float16, device="cuda")
    B.chunk_attn(cfg, cache, xd[:, :8], starts, 700, out, B.make_chunk_workspace(cfg, 700, 700))
    torch.cuda.synchronize()
    want, tol = attention64(x[:, :8], x[:, 8:16], x[:, 16:], 0, cfg.sm_scale)
    check_attention(out, want, tol)


def test_tokens_far_apart():
    """Rows 2^23 elements apart, the last of them more than 4 GB from the first."""
    n, stride = 270, 1 << 23
    cfg = B.make_config(2, 2, 1, 512, BF16)
    mem = torch.empty((n - 1) * stride + 4 * D, dtype=torch.bfloat16, device="cuda")
    x = mem.as_strided((n, 4, D), (stride, D, 1))
    host = randn((n, 4, D), BF16, 93)
    x.copy_(host)
    lens = [200, 70]
    out = torch.zeros(n, 2, D, dtype=torch.bfloat16, device="cuda")
    B.prefill_attn(cfg, x[:, :2], x[:, 2:3], x[:, 3:], i32(starts_of(lens)), 200, out)
    cache = make_cache(cfg, [0, 0], [0, 0], BF16, 0, 94)[1]
    B.append_chunk(cfg, cache, x[:, 2:3], x[:, 3:], i32(starts_of(lens)), 200)
    torch.cuda.synchronize()
    at = 0
    for b, m in enumerate(lens):
        want, tol = attention64(host[at:at + m, :2], host[at:at + m, 2:3], host[at:at + m, 3:], 0, cfg.sm_scale)
        check_attention(out[at:at + m], want, tol)
        assert torch.equal(cache.k[b, :m].cpu(), host[at:at + m, 2]) and torch.equal(cache.v[b, :m].cpu(), host[at:at + m, 3])
        at += m
