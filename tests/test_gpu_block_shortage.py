"""A pool that runs out of blocks: the step does not take place, neither in the block table nor in the calls enqueued behind it."""
import numpy as np
import pytest
import torch

from paper_2508_08256_amd import binding as B
from prompt_util import D, block_table_plain, starts_of
from test_gpu_prompt_cache import empty_cache, i32, randn, table_case

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("batch,before", [(1, [0, 7]), (3, [0, 5, 9, 9]), (3, [-4, 100, -7, 1 << 30]), (700, None)])
def test_offsets_say_that_no_sequence_grows(batch, before):
    """Whatever the offsets held before; a negative counter passed on stays one and costs no block."""
    before = starts_of([3] * batch) if before is None else np.array(before, np.int32)
    cfg = B.make_config(batch, 1, 1, 256, B.F16)
    old, new = np.full(batch, 70), np.full(batch, 130)
    table, free = table_case(batch, 256, 64, old, batch - 1, 1)
    new_ends = new.copy()
    new_ends[0] = 0  # gives two blocks back: enough for the others
    t, f, out, s, slots = i32(table), i32(free), i32([-77]), i32(before), torch.full((60 * batch,), -6, dtype=torch.int32, device="cuda")

    def step(lens, n_free):
        B.block_table(cfg, 64, i32(old), i32(lens), t, f, i32([n_free]), out, s, slots)
        torch.cuda.synchronize()
        return int(out)

    def untouched():
        return (np.array_equal(t.cpu().numpy(), table) and np.array_equal(f.cpu().numpy(), free)
                and bool((slots == -6).all()) and s.tolist() == [int(before[0])] * (batch + 1))

    assert step(new, batch - 1) == -1 and untouched()
    for lens in (new, new_ends, np.zeros(batch, np.int64)):  # also where blocks would come back
        assert step(lens, -1) == -1 and untouched()
    left, want, free_after, starts, where = block_table_plain(64, 256, old, new_ends, table, free, batch - 1)
    assert step(new_ends, batch - 1) == left >= 0
    assert np.array_equal(t.cpu().numpy(), want) and np.array_equal(f.cpu().numpy(), free_after)
    assert s.tolist() == starts.tolist() and slots.tolist()[: len(where)] == where.tolist()


@pytest.mark.parametrize("captured", [False, True])
def test_nothing_is_written_behind_a_table_that_fell_short(captured):
    """Table, append and attention on one stream, the pool one block too small: rows, codes and outputs stay, a call from the same
    lengths and counter works once a sequence has ended."""
    nb, hq, hkv, cap, bt = 3, 4, 2, 512, 64
    cfg = B.make_config(nb, hq, hkv, cap, B.BF16)
    cache = empty_cache(cfg, [0] * nb, B.BF16, bt)
    n_pool = 6
    cache.block_table.fill_(0)  # entries not in use name a block of the pool: writes through them would show
    free, counts = i32(np.arange(n_pool - 1, -1, -1)), [i32([n_pool]), i32([0])]
    lens, after, starts = cache.seq_lens, i32([0] * nb), i32([0] * (nb + 1))
    rows, width = 300, 200
    x = randn((rows, hq + 2 * hkv, D), B.BF16, 1).cuda()
    out = torch.zeros(rows, hq, D, dtype=torch.bfloat16, device="cuda")
    ws = B.make_chunk_workspace(cfg, rows, width)

    def step(a, b):
        B.block_table(cfg, bt, lens, after, cache.block_table, free, a, b, starts)
        B.append_chunk(cfg, cache, x[:, hq:hq + hkv], x[:, hq + hkv:], starts, width)
        B.chunk_attn(cfg, cache, x[:, :hq], starts, width, out, ws)

    graphs = []
    if captured:
        step(counts[0], i32([0]))  # nothing grows yet
        torch.cuda.synchronize()
        for k in range(2):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[k]):
                step(counts[k], counts[1 - k])

    def run(lengths, at):
        after.copy_(i32(lengths))
        out.fill_(7.0)
        if captured:
            graphs[at].replay()
        else:
            step(counts[at], counts[1 - at])
        torch.cuda.synchronize()
        return int(counts[1 - at])

    def state():
        return [t.clone() for t in (cache.k, cache.v, cache.kbits, cache.kmeta, cache.kabsmax, cache.block_table, free)]

    assert run([100, 60, 64], 0) == 2  # blocks 0 .. 3
    lens.copy_(after)
    before = state()
    assert run([200, 70, 64], 1) == -1  # three more of two
    assert int(counts[1]) == 2
    assert all(torch.equal(a, b) for a, b in zip(state(), before)) and bool((out == 7.0).all())
    assert run([200, 0, 64], 0) == -1  # the counter that fell short, by mistake: nothing is lost
    assert all(torch.equal(a, b) for a, b in zip(state(), before)) and bool((out == 7.0).all())
    counts[1].fill_(2)
    assert run([200, 0, 64], 1) == 1  # the second sequence has ended
    assert starts.tolist() == [0, 100, 100, 100]
    assert bool((out[100:] == 7.0).all()) and not bool((out[:100] == 7.0).all(dim=2).any())
    k = cache.k[cache.block_table[0].long()].transpose(0, 1).reshape(hkv, cap, D)
    assert torch.equal(k[:, 100:200], x[:100, hq:hq + hkv].transpose(0, 1))
    assert sorted(cache.block_table[0, :4].tolist() + cache.block_table[2, :1].tolist() + free[:1].tolist()) == list(range(n_pool))
