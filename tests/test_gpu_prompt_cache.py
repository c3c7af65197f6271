"""Chunks into the cache and its 1-bit copy, block tables, and both together with attention and the decode step."""
import numpy as np
import pytest
import torch

from paper_2508_08256_amd import binding as B
from prompt_util import D, attention64, block_table_plain, check_attention, starts_of, tdtype

pytestmark = pytest.mark.gpu
F16, BF16 = B.F16, B.BF16


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def i32(a):
    return torch.as_tensor(np.asarray(a, np.int32), device="cuda")


def randn(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(tdtype(dtype))


def empty_cache(cfg, lens, dtype, block_tokens, seed=0):
    nb, hkv, cap = cfg.batch, cfg.n_kv_heads, cfg.max_ctx
    if not block_tokens:
        k, v = (torch.zeros(nb * hkv, cap, D, dtype=tdtype(dtype), device="cuda") for _ in range(2))
        return B.DeviceCache(cfg, k, v, i32(lens))
    per = cap // block_tokens
    table = torch.randperm(nb * per + 2, generator=torch.Generator().manual_seed(seed))[: nb * per].view(nb, per)
    k, v = (torch.zeros(nb * per + 2, hkv, block_tokens, D, dtype=tdtype(dtype), device="cuda") for _ in range(2))
    return B.DeviceCache(cfg, k, v, i32(lens), table.to(torch.int32).cuda())


def logical(cache, pool):
    """[batch][kv heads][max_ctx][D] of a cache's K or V."""
    cfg = cache.cfg
    if cache.block_table is None:
        return pool.view(cfg.batch, cfg.n_kv_heads, cfg.max_ctx, D).cpu()
    return pool[cache.block_table.long()].transpose(1, 2).reshape(cfg.batch, cfg.n_kv_heads, cfg.max_ctx, D).cpu()


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("g", [32, 64, 128, 256])
@pytest.mark.parametrize("block_tokens", [0, 256])
def test_chunk_by_chunk_equals_the_bulk_quantizer(dtype, g, block_tokens):
    """Several chunks of unequal sequences, none and one token among them, boundaries anywhere in groups and pair blocks: rows,
    codes and (s, z) are those of one bulk quantization, bit for bit, and what no chunk touches stays."""
    cfg = B.make_config(4, 2, 2, 1024, dtype, group_size=g)
    chunks = [[1, 0, 64, 300], [31, 33, 1, 211], [0, 200, 63, 1], [97, 64, 129, 256], [1, 1, 0, 255]]
    cache = empty_cache(cfg, [0] * 4, dtype, block_tokens)
    K, V = (torch.zeros(4, 2, 1024, D, dtype=tdtype(dtype)) for _ in range(2))
    lens = np.zeros(4, np.int64)
    for c, new in enumerate(chunks):
        n = sum(new)
        # views of a fused product with three rows of padding
        qkv = randn((n + 3, 6, D), dtype, 100 + c) * (1 + c)
        k, v = qkv[:, 2:4], qkv[:, 4:]
        at = 0
        for b in range(4):
            K[b, :, lens[b]:lens[b] + new[b]] = k[at:at + new[b]].transpose(0, 1)
            V[b, :, lens[b]:lens[b] + new[b]] = v[at:at + new[b]].transpose(0, 1)
            at += new[b]
        dev = qkv.cuda()
        B.append_chunk(cfg, cache, dev[:, 2:4], dev[:, 4:], i32(starts_of(new)), max(new))
        lens += new
        cache.seq_lens.copy_(i32(lens))
        torch.cuda.synchronize()
        assert torch.equal(logical(cache, cache.k), K) and torch.equal(logical(cache, cache.v), V)
        bulk = B.DeviceCache(cfg, K.view(8, 1024, D).cuda(), V.view(8, 1024, D).cuda(), i32(lens))
        B.quantize_keys(cfg, bulk)
        torch.cuda.synchronize()
        assert torch.equal(cache.kbits, bulk.kbits) and torch.equal(cache.kmeta, bulk.kmeta), c
        assert bool((cache.kabsmax >= bulk.kabsmax).all())
        if c == 0:
            assert torch.equal(cache.kabsmax, bulk.kabsmax)


@pytest.mark.parametrize("dtype,n_kv,new", [(F16, 4, [5000, 63]), (BF16, 8, [1, 2500])])
def test_whole_prompts_into_an_empty_cache(dtype, n_kv, new):
    cfg = B.make_config(2, n_kv, n_kv, 5056, dtype)
    cache = empty_cache(cfg, [0, 0], dtype, 64)
    n = sum(new)
    k, v = randn((n, n_kv, D), dtype, 1).cuda(), randn((n, n_kv, D), dtype, 2).cuda()
    B.append_chunk(cfg, cache, k, v, i32(starts_of(new)), max(new))
    cache.seq_lens.copy_(i32(new))
    flat = [torch.zeros(2 * n_kv, 5056, D, dtype=k.dtype, device="cuda") for _ in range(2)]
    for t, x in zip(flat, (k, v)):
        t.view(2, n_kv, 5056, D)[0, :, : new[0]] = x[: new[0]].transpose(0, 1)
        t.view(2, n_kv, 5056, D)[1, :, : new[1]] = x[new[0]:].transpose(0, 1)
    bulk = B.DeviceCache(cfg, *flat, i32(new))
    B.quantize_keys(cfg, bulk)
    torch.cuda.synchronize()
    for a, b in ((cache.kbits, bulk.kbits), (cache.kmeta, bulk.kmeta), (cache.kabsmax, bulk.kabsmax)):
        assert torch.equal(a, b)
    assert torch.equal(logical(cache, cache.k).view(-1), bulk.k.cpu().view(-1))
    assert torch.equal(logical(cache, cache.v).view(-1), bulk.v.cpu().view(-1))


def test_a_chunk_past_the_capacity_and_bad_offsets():
    """The rows that fit are written, the rest left out; nothing outside the arrays is touched whatever the offsets say."""
    cfg = B.make_config(3, 1, 1, 128, F16)
    cache = empty_cache(cfg, [120, 128, 5], F16, 0)
    guard = cache.k.clone()
    k, v = randn((40, 1, D), F16, 3).cuda(), randn((40, 1, D), F16, 4).cuda()
    B.append_chunk(cfg, cache, k, v, i32([0, 20, 30, 1 << 30]), 20)
    torch.cuda.synchronize()
    assert torch.equal(cache.k[0, 120:], k[:8, 0]) and torch.equal(cache.v[0, 120:], v[:8, 0])
    assert torch.equal(cache.k[0, :120], guard[0, :120]) and torch.equal(cache.k[1], guard[1])
    assert torch.equal(cache.k[2, 5:15], k[30:, 0]) and torch.equal(cache.k[2, 15:], guard[2, 15:])
    before = cache.k.clone()
    B.append_chunk(cfg, cache, k, v, i32([30, 20, -7, -9]), 20)  # sequences of no tokens
    torch.cuda.synchronize()
    assert torch.equal(cache.k, before)


def test_one_token_chunks_equal_the_append_call():
    cfg = B.make_config(3, 4, 2, 512, BF16, group_size=64)
    lens = [0, 63, 200]
    caches = [empty_cache(cfg, lens, BF16, 0) for _ in range(2)]
    rows = [randn((6, 512, D), BF16, 5).cuda(), randn((6, 512, D), BF16, 6).cuda()]
    k, v = randn((3, 2, D), BF16, 7).cuda(), randn((3, 2, D), BF16, 8).cuda()
    for c in caches:
        c.k.copy_(rows[0]), c.v.copy_(rows[1])
        B.quantize_keys(cfg, c)
    B.append_key(cfg, caches[0], k, v)
    B.append_chunk(cfg, caches[1], k, v, i32([0, 1, 2, 3]), 1)
    torch.cuda.synchronize()
    for name in ("k", "v", "kbits", "kmeta", "kabsmax"):
        assert torch.equal(getattr(caches[0], name), getattr(caches[1], name)), name


# ---- block tables -------------------------------------------------------------------------------------------------------


def table_case(batch, max_ctx, bt, old, spare, seed):
    rng = np.random.default_rng(seed)
    old = np.asarray(old)
    held = -(-np.clip(old, 0, max_ctx) // bt)
    n_blocks = int(held.sum()) + spare
    perm = rng.permutation(n_blocks).astype(np.int32)
    table = rng.integers(-9, 0, (batch, max_ctx // bt)).astype(np.int32)  # entries not in use: anything
    at = 0
    for b in range(batch):
        table[b, : held[b]] = perm[at:at + held[b]]
        at += held[b]
    free = np.full(n_blocks, -1, np.int32)
    free[:spare] = perm[at:]
    return table, free


def run_table(cfg, bt, old, new, table, free, n_free, n_slots):
    d = dict(table=i32(table), free=i32(free), out=i32([-77]), starts=torch.full((cfg.batch + 1,), -5, dtype=torch.int32, device="cuda"),
             slots=torch.full((n_slots,), -6, dtype=torch.int32, device="cuda"))
    nf, o, w = i32([n_free]), i32(old), i32(new)
    for _ in range(2):  # it may be repeated
        B.block_table(cfg, bt, o, w, d["table"], d["free"], nf, d["out"], d["starts"], d["slots"])
    torch.cuda.synchronize()
    return {k: v.cpu().numpy() for k, v in d.items()}


def check_table(cfg, bt, old, new, table, free, n_free, n_slots=None):
    left, t, f, starts, slots = block_table_plain(bt, cfg.max_ctx, np.asarray(old), np.asarray(new), table, free, n_free)
    n_slots = (0 if slots is None else len(slots)) + 3 if n_slots is None else n_slots
    got = run_table(cfg, bt, old, new, table, free, n_free, n_slots)
    assert got["out"][0] == left
    assert np.array_equal(got["table"], t) and np.array_equal(got["free"], f)
    if left < 0:
        assert (got["starts"] == -5).all() and (got["slots"] == -6).all()
        return
    assert np.array_equal(got["starts"], starts)
    n = min(n_slots, len(slots))
    assert np.array_equal(got["slots"][:n], slots[:n]) and (got["slots"][n:] == -6).all()


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("batch,max_ctx,bt", [(1, 64, 64), (5, 1024, 64), (70, 4096, 128), (300, 65536, 64), (600, 2048, 256)])
def test_block_table(batch, max_ctx, bt, seed):
    """Growth, shrinking, ends and starts in one call, around the block boundaries, against a list as a stack."""
    rng = np.random.default_rng([seed, batch])
    old = rng.integers(0, max_ctx // 2 + 1, batch)
    new = np.clip(old + rng.integers(-2 * bt, 2 * bt + 1, batch), 0, max_ctx)
    kind = rng.integers(0, 8, batch)
    new[kind == 0] = 0
    new[kind == 1] = np.minimum(old + 1, max_ctx)[kind == 1]
    old[kind == 2] = 0
    new[kind == 3] = (new // bt * bt)[kind == 3]
    new[kind == 4] = max_ctx if seed == 1 else (old // bt * bt)[kind == 4]
    cfg = B.make_config(batch, 2, 1, max_ctx, F16, group_size=64)
    need = int((-(-new // bt) + old // -bt).sum())
    for spare in {max(0, need), max(0, need) + 1, abs(need) + 50, max(0, need - 1)}:
        table, free = table_case(batch, max_ctx, bt, old, spare, seed)
        check_table(cfg, bt, old, new, table, free, spare)


def test_block_table_lengths_out_of_range_and_few_slots():
    cfg = B.make_config(3, 1, 1, 256, F16)
    table, free = table_case(3, 256, 64, [10, 300, -3], 9, 1)
    check_table(cfg, 64, [10, 300, -3], [1000, 256, 100], table, free, 9, n_slots=200)
    check_table(cfg, 64, [10, 300, -3], [-1, -5, -9], table, free, 9)


def test_block_table_of_the_largest_batch():
    """16384 sequences: their sums fill 64 KiB of shared memory."""
    n = 16384
    rng = np.random.default_rng(5)
    old, new = rng.integers(0, 257, n), rng.integers(0, 257, n)
    cfg = B.make_config(n, 1, 1, 256, F16)
    spare = max(0, int((-(-new // 64) + old // -64).sum())) + 7
    table, free = table_case(n, 256, 64, old, spare, 6)
    check_table(cfg, 64, old, new, table, free, spare)


def test_block_table_without_offsets():
    cfg = B.make_config(2, 1, 1, 256, F16)
    table, free = table_case(2, 256, 64, [10, 64], 4, 2)
    left, t, f, _, _ = block_table_plain(64, 256, np.array([10, 64]), np.array([70, 65]), table, free, 4)
    td, fd, out = i32(table), i32(free), i32([0])
    B.block_table(cfg, 64, i32([10, 64]), i32([70, 65]), td, fd, i32([4]), out)
    torch.cuda.synchronize()
    assert int(out) == left and np.array_equal(td.cpu().numpy(), t) and np.array_equal(fd.cpu().numpy(), f)


# ---- all of it as a server runs it -----------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype,captured", [(BF16, False), (F16, True)])
def test_prompts_chunk_by_chunk_then_decode(dtype, captured):
    """Blocks handed out from lengths, chunks appended and attended over, drafts taken back, then decode steps: the outputs
    are those of one attention over each whole prompt, and the decode steps those on a cache quantized in bulk.  Eagerly, and
    with every step replayed from a graph."""
    nb, hq, hkv, cap, bt = 3, 8, 2, 1024, 64
    cfg = B.make_config(nb, hq, hkv, cap, dtype)
    chunks = [[300, 1, 0], [129, 64, 5], [0, 2, 600], [7, 300, 3]]
    total = np.sum(chunks, axis=0)
    n_pool = 3 * cap // bt
    cache = empty_cache(cfg, [0] * nb, dtype, bt)
    table = cache.block_table
    table.fill_(0)
    free = torch.randperm(n_pool, generator=torch.Generator().manual_seed(1)).to(torch.int32).cuda()
    counts, at = [i32([n_pool]), i32([0])], 0
    toks = [randn((int(total[b]) + 4, hq + 2 * hkv, D), dtype, 200 + b) for b in range(nb)]
    lens, after, starts = i32([0] * nb), i32([0] * nb), i32([0] * (nb + 1))
    rows, width = 1000, 600
    slots = torch.zeros(rows, dtype=torch.int32, device="cuda")
    x = torch.zeros(rows, hq + 2 * hkv, D, dtype=tdtype(dtype), device="cuda")
    out = torch.zeros(rows, hq, D, dtype=tdtype(dtype), device="cuda")
    ws = B.make_chunk_workspace(cfg, rows, width)

    def step(nf, nf_out):
        B.block_table(cfg, bt, lens, after, table, free, nf, nf_out, starts, slots)
        B.append_chunk(cfg, cache, x[:, hq:hq + hkv], x[:, hq + hkv:], starts, width)
        B.chunk_attn(cfg, cache, x[:, :hq], starts, width, out, ws)

    cache.seq_lens.zero_()
    graphs = []
    if captured:
        for k in range(2):
            step(counts[k], i32([0]))  # nothing grows yet
            torch.cuda.synchronize()
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[k]):
                step(counts[k], counts[1 - k])
    done = np.zeros(nb, np.int64)
    outs = [[] for _ in range(nb)]
    for new in chunks:
        x.fill_(float("nan"))
        lo = 0
        for b in range(nb):
            x[lo:lo + new[b]] = toks[b][done[b]:done[b] + new[b]].cuda()
            lo += new[b]
        after.copy_(i32(done + new))
        if captured:
            graphs[at].replay()
        else:
            step(counts[at], counts[1 - at])
        torch.cuda.synchronize()
        at = 1 - at
        lo = 0
        for b in range(nb):
            outs[b].append(out[lo:lo + new[b]].cpu())
            lo += new[b]
        want_slots = [int(table[b, p // bt]) * bt + p % bt for b in range(nb) for p in range(done[b], done[b] + new[b])]
        assert slots[:lo].tolist() == want_slots
        for t, p in list(enumerate(want_slots))[:: max(1, lo // 20)]:  # the slots say where the rows went
            assert torch.equal(cache.k[p // bt, :, p % bt], x[t, hq:hq + hkv])
        done += new
        lens.copy_(after)
        cache.seq_lens.copy_(after)
        assert int(counts[at]) == n_pool - int((-(-done // bt)).sum())
    for b in range(nb):
        t = toks[b][: total[b]]
        want, tol = attention64(t[:, :hq], t[:, hq:hq + hkv], t[:, hq + hkv:], 0, cfg.sm_scale)
        check_attention(torch.cat(outs[b]), want, tol, f"sequence {b}")
    # four drafted tokens are taken back: lengths shrink, blocks come back; then the same tokens as decode steps
    after.copy_(i32(done + 4))
    B.block_table(cfg, bt, lens, after, table, free, counts[at], counts[1 - at], starts)
    B.block_table(cfg, bt, after, lens, table, free, counts[1 - at], counts[at])
    flat = [torch.zeros(nb * hkv, cap, D, dtype=tdtype(dtype), device="cuda") for _ in range(2)]
    for b in range(nb):
        for which in (0, 1):
            t = toks[b][: total[b], hq + which * hkv:hq + (which + 1) * hkv]
            flat[which].view(nb, hkv, cap, D)[b, :, : total[b]] = t.transpose(0, 1).cuda()
    bulk = B.DeviceCache(cfg, *flat, cache.seq_lens)
    B.quantize_keys(cfg, bulk)
    budgets, wsd = i32([100] * nb), B.make_workspace(cfg, 100)
    for i in range(4):
        B.block_table(cfg, bt, lens, lens + 1, table, free, counts[at], counts[1 - at])
        at = 1 - at
        new = torch.stack([toks[b][total[b] + i] for b in range(nb)]).cuda()
        got = []
        for c in (cache, bulk):
            o = torch.zeros(1, nb, hq, D, device="cuda")
            B.decode_step(cfg, [c], new[None, :, :hq].contiguous(), new[None, :, hq:hq + hkv].contiguous(),
                          new[None, :, hq + hkv:].contiguous(), budgets, 100, o, None, None, wsd)
            got.append(o)
        torch.cuda.synchronize()
        assert float((got[0] - got[1]).abs().max()) <= 1e-5
        lens.add_(1)
        cache.seq_lens.add_(1)
    # every block is somewhere exactly once
    held = (-(-(lens.cpu().numpy()) // bt))
    used = [int(table[b, e]) for b in range(nb) for e in range(held[b])]
    assert sorted(used + free[: int(counts[at])].tolist()) == list(range(n_pool))
