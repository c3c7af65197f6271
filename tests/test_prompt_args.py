"""Refusals of the calls that take many new tokens per sequence: on the host, before anything is launched."""
import ctypes as C
import math
import types

import pytest
import torch

from paper_2508_08256_amd import binding as B

CACHE = B.Cache(0x1000, 0x2000, 0x3000, 0x4000, 0x4800, 0x5000)
BIG = 1 << 40


def prefill(cfg, q=0x6000, qs=512, k=0x7000, ks=256, v=0x8000, vs=256, starts=0x9000, n=10, most=10, out=0xA000):
    return B.lib().fier_prefill_attn(C.byref(cfg), q, qs, k, ks, v, vs, starts, n, most, out, None)


def chunk(cfg, cache=CACHE, q=0x6000, qs=512, starts=0x9000, n=10, most=10, out=0xA000, ws=0x100000, size=BIG):
    return B.lib().fier_chunk_attn(C.byref(cfg), C.byref(cache), q, qs, starts, n, most, out, ws, size, None)


def append(cfg, cache=CACHE, k=0x7000, ks=256, v=0x8000, vs=256, starts=0x9000, n=10, most=10):
    return B.lib().fier_append_chunk(C.byref(cfg), C.byref(cache), k, ks, v, vs, starts, n, most, None)


@pytest.fixture
def cfg():
    return B.make_config(2, 4, 2, 256, B.BF16)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), B.EINVAL), (dict(k=None), B.EINVAL), (dict(v=None), B.EINVAL), (dict(out=None), B.EINVAL),
    (dict(starts=None), B.EINVAL), (dict(n=-1), B.EINVAL), (dict(most=-1), B.EINVAL), (dict(n=(1 << 24) + 1), B.ESHAPE),
    (dict(qs=511), B.ESHAPE), (dict(qs=516), B.EALIGN), (dict(ks=248), B.ESHAPE), (dict(vs=-256), B.ESHAPE),
    (dict(vs=260), B.EALIGN), (dict(q=0x6008), B.EALIGN), (dict(k=0x7002), B.EALIGN), (dict(v=0x8004), B.EALIGN),
    (dict(out=0xA008), B.EALIGN), (dict(starts=0x9002), B.EALIGN)])
def test_prefill_refusals(cfg, change, status):
    assert prefill(cfg, **change) == status


@pytest.mark.parametrize("change,status", [
    (dict(q=None), B.EINVAL), (dict(out=None), B.EINVAL), (dict(starts=None), B.EINVAL), (dict(n=-1), B.EINVAL),
    (dict(qs=504), B.ESHAPE), (dict(q=0x6004), B.EALIGN), (dict(out=0xA004), B.EALIGN), (dict(ws=None), B.EWORKSPACE),
    (dict(size=0), B.EWORKSPACE), (dict(ws=0x100010), B.EALIGN), (dict(cache=B.Cache(0, 0, 0, 0, 0, 0)), B.EINVAL),
    (dict(cache=B.Cache(0x1000, 0x2000, 0x3000, 0x4000, 0x4800, 0x5000, 0x6000, 96)), B.ESHAPE)])
def test_chunk_refusals(cfg, change, status):
    assert chunk(cfg, **change) == status


def test_the_chunk_workspace_size_is_checked(cfg):
    for c, n, most in ((cfg, 10, 10), (cfg, 300, 7), (B.make_config(16, 32, 8, 65600, B.BF16), 16, 1)):
        need = B.chunk_workspace_bytes(c, n, most)
        assert need > 0 and need % 256 == 0
        assert chunk(c, qs=4096, n=n, most=most, size=need - 1) == B.EWORKSPACE
    assert B.chunk_workspace_bytes(cfg, -1, 1) == 0 and B.chunk_workspace_bytes(cfg, 1, -1) == 0
    assert B.chunk_workspace_bytes(B.make_config(2, 5, 2, 256), 1, 1) == 0
    # a call for fewer tokens needs no more than the workspace made for many
    c = B.make_config(4, 32, 8, 32768, B.BF16)
    sizes = [B.chunk_workspace_bytes(c, n, m) for n, m in ((4, 1), (16, 4), (64, 16), (600, 512), (4096, 4096), (1 << 20, 1 << 20))]
    assert max(sizes) <= 256 << 20


@pytest.mark.parametrize("change,status", [
    (dict(k=None), B.EINVAL), (dict(v=None), B.EINVAL), (dict(starts=None), B.EINVAL), (dict(most=-3), B.EINVAL),
    (dict(ks=255), B.ESHAPE), (dict(ks=257), B.EALIGN), (dict(vs=128), B.ESHAPE), (dict(k=0x7001), B.EALIGN),
    (dict(cache=B.Cache(0x1000, 0x2008, 0x3000, 0x4000, 0x4800, 0x5000)), B.EALIGN)])
def test_append_refusals(cfg, change, status):
    assert append(cfg, **change) == status


def test_configurations_are_checked_first():
    for bad, status in ((B.make_config(2, 4, 2, 256, head_dim=64), B.EUNSUPPORTED), (B.make_config(2, 18, 2, 256), B.EUNSUPPORTED),
                        (B.make_config(2, 4, 2, 250), B.ESHAPE), (B.make_config(0, 4, 2, 256), B.EINVAL)):
        assert prefill(bad) == chunk(bad) == append(bad) == status
    for scale in (math.inf, -math.inf):
        c = B.make_config(2, 4, 2, 256, sm_scale=scale)
        assert prefill(c) == chunk(c) == B.EINVAL


def test_no_tokens_are_no_launch(cfg):
    """Nothing to do: accepted, and nothing is enqueued (there is not even a GPU here)."""
    for kw in (dict(n=0), dict(most=0)):
        assert prefill(cfg, **kw) == chunk(cfg, **kw) == append(cfg, **kw) == B.OK


def table(cfg, bt=64, old=0x1000, new=0x2000, tab=0x3000, free=0x4000, n_blocks=8, nf=0x5000, nfo=0x5004, starts=0x6000,
          slots=0x7000, n_slots=4):
    return B.lib().fier_block_table(C.byref(cfg), bt, old, new, tab, free, n_blocks, nf, nfo, starts, slots, n_slots, None)


@pytest.mark.parametrize("change,status", [
    (dict(old=None), B.EINVAL), (dict(new=None), B.EINVAL), (dict(tab=None), B.EINVAL), (dict(free=None), B.EINVAL),
    (dict(nf=None), B.EINVAL), (dict(nfo=None), B.EINVAL), (dict(nfo=0x5000), B.EINVAL), (dict(new=0x1000), B.EINVAL),
    (dict(n_blocks=-1), B.EINVAL), (dict(n_slots=-1), B.EINVAL), (dict(starts=None), B.EINVAL), (dict(slots=None), B.EINVAL),
    (dict(bt=0), B.ESHAPE), (dict(bt=32), B.ESHAPE), (dict(bt=192), B.ESHAPE), (dict(bt=512), B.ESHAPE),
    (dict(n_blocks=1 << 25), B.ESHAPE), (dict(tab=0x3002), B.EALIGN), (dict(slots=0x7001), B.EALIGN), (dict(nf=0x5001), B.EALIGN)])
def test_block_table_refusals(cfg, change, status):
    assert table(cfg, **change) == status


def test_block_table_sizes():
    assert table(B.make_config(16385, 1, 1, 256)) == B.ESHAPE
    assert table(B.make_config(4096, 1, 1, 1 << 20)) == B.ESHAPE
    assert table(B.make_config(2, 1, 1, 256, group_size=128), bt=64) == B.ESHAPE


def test_the_binding_refuses_other_layouts(monkeypatch):
    monkeypatch.setattr(B, "_stream", lambda: None)
    cfg = B.make_config(2, 4, 2, 256, B.BF16)
    q, k = torch.zeros(10, 4, 128, dtype=torch.bfloat16), torch.zeros(10, 2, 128, dtype=torch.bfloat16)
    starts = torch.zeros(3, dtype=torch.int32)
    wide = torch.zeros(10, 8, 128, dtype=torch.bfloat16)
    for bad in (dict(q=q[:, :3]), dict(q=q.float()), dict(k=k[:9]), dict(v=wide[:, ::4]), dict(out=wide[:, :4]), dict(q=q.transpose(0, 1))):
        kw = dict(dict(q=q, k=k, v=k, out=q), **bad)
        with pytest.raises(B.FierError) as e:
            B.prefill_attn(cfg, kw["q"], kw["k"], kw["v"], starts, 5, kw["out"])
        assert e.value.status == B.ESHAPE
    cache, ws = types.SimpleNamespace(c=CACHE), torch.zeros(64, dtype=torch.uint8)
    with pytest.raises(B.FierError) as e:
        B.chunk_attn(cfg, cache, q, starts, 5, q, ws)
    assert e.value.status == B.EWORKSPACE
    with pytest.raises(B.FierError):
        B.append_chunk(cfg, cache, k, wide[:, :3], starts, 5)
    i = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    good = [i(2), i(2), i(8), i(9), i(1), i(1), i(3), i(4)]
    for at, bad in ((0, i(3)), (2, i(9)), (6, i(2)), (3, torch.zeros(9, dtype=torch.int64)), (7, i(8)[::2])):
        args = list(good)
        args[at] = bad
        with pytest.raises(B.FierError):
            B.block_table(cfg, 64, *args)


@pytest.mark.parametrize("starts", [torch.zeros(3, dtype=torch.int64), torch.zeros(2, dtype=torch.int32),
                                    torch.zeros(6, dtype=torch.int32)[::2]])
def test_the_binding_refuses_other_offsets(monkeypatch, starts):
    """torch's sums of int32 lengths have 64 bits: read as 32-bit offsets they would be other sequences."""
    monkeypatch.setattr(B, "_stream", lambda: None)
    cfg, cache = B.make_config(2, 4, 2, 256, B.BF16), types.SimpleNamespace(c=CACHE)
    q, k = torch.zeros(10, 4, 128, dtype=torch.bfloat16), torch.zeros(10, 2, 128, dtype=torch.bfloat16)
    ws = torch.zeros(64, dtype=torch.uint8)
    for call in (lambda: B.prefill_attn(cfg, q, k, k, starts, 0, q), lambda: B.append_chunk(cfg, cache, k, k, starts, 0),
                 lambda: B.chunk_attn(cfg, cache, q, starts, 0, q, ws)):
        with pytest.raises(B.FierError) as e:
            call()
        assert e.value.status == B.ESHAPE
