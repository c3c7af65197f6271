"""Bounds of the calls that take many new tokens per sequence, on the host."""
import math
import types

import pytest
import torch

from paper_2508_08256_amd import binding as B
from test_prompt_args import CACHE, append, chunk, prefill


@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_a_softmax_scale_that_has_no_logarithmic_form_is_refused(sign):
    """The kernels take sm_scale * log2(e): an infinity from 2^128 / log2(e) = 2.36e38 on."""
    for scale, status in ((2.35e38, B.OK), (2.37e38, B.EINVAL), (3.4e38, B.EINVAL), (math.inf, B.EINVAL)):
        c = B.make_config(2, 4, 2, 256, sm_scale=sign * scale)
        assert prefill(c, n=0) == chunk(c, n=0) == status, scale  # no tokens: nothing is launched
        assert append(c, n=0) == B.OK  # has no use for it


def _args(dtype=torch.bfloat16):
    q, k = torch.zeros(10, 4, 128, dtype=dtype), torch.zeros(10, 2, 128, dtype=dtype)
    return q, k, torch.zeros(3, dtype=torch.int32), torch.zeros(1 << 16, dtype=torch.uint8)


def _calls(cfg, q, k, v, starts, out, ws):
    """No sequence may have tokens: what is not refused launches nothing."""
    cache = types.SimpleNamespace(c=CACHE)
    return [lambda: B.prefill_attn(cfg, q, k, v, starts, 0, out), lambda: B.chunk_attn(cfg, cache, q, starts, 0, out, ws),
            lambda: B.append_chunk(cfg, cache, k, v, starts, 0)]


@pytest.mark.parametrize("dtype", [torch.float16, torch.int16])
@pytest.mark.parametrize("at", ["q", "k", "v", "out"])
def test_the_binding_refuses_rows_of_another_type(monkeypatch, dtype, at):
    """Two bytes are not enough: fp16 rows read as bf16 give numbers without an error."""
    monkeypatch.setattr(B, "_stream", lambda: None)
    cfg = B.make_config(2, 4, 2, 256, B.BF16)
    q, k, starts, ws = _args()
    kw = dict(q=q, k=k, v=k, out=q)
    kw[at] = kw[at].to(dtype)
    takes = {"q": (0, 1), "k": (0, 2), "v": (0, 2), "out": (0, 1)}[at]
    for i, call in enumerate(_calls(cfg, kw["q"], kw["k"], kw["v"], starts, kw["out"], ws)):
        if i in takes:
            with pytest.raises(B.FierError) as e:
                call()
            assert e.value.status == B.ESHAPE


def test_the_binding_refuses_offsets_of_another_type(monkeypatch):
    monkeypatch.setattr(B, "_stream", lambda: None)
    cfg = B.make_config(2, 4, 2, 256, B.BF16)
    q, k, _, ws = _args()
    for call in _calls(cfg, q, k, k, torch.zeros(3), q, ws):  # float32: four bytes as well
        with pytest.raises(B.FierError) as e:
            call()
        assert e.value.status == B.ESHAPE
    good = [torch.zeros(n, dtype=torch.int32) for n in (2, 2, 8, 9, 1, 1, 3, 4)]
    for at in range(8):
        args = list(good)
        args[at] = args[at].float()
        with pytest.raises(B.FierError) as e:
            B.block_table(cfg, 64, *args)
        assert e.value.status == B.EINVAL


def test_the_binding_refuses_tensors_in_host_memory(monkeypatch):
    """Nothing else is wrong with them; a kernel would fault on their addresses."""
    monkeypatch.setattr(B, "_stream", lambda: None)
    cfg = B.make_config(2, 4, 2, 256, B.BF16)
    q, k, starts, ws = _args()
    for call, status in zip(_calls(cfg, q, k, k, starts, q, ws), (B.EINVAL, B.EWORKSPACE, B.EINVAL)):
        with pytest.raises(B.FierError) as e:
            call()
        assert e.value.status == status
    with pytest.raises(B.FierError) as e:
        B.block_table(cfg, 64, *(torch.zeros(n, dtype=torch.int32) for n in (2, 2, 8, 9, 1, 1, 3, 4)))
    assert e.value.status == B.EINVAL


@pytest.mark.parametrize("n_q,n_kv", [(1, 1), (8, 8), (12, 4), (32, 8), (7, 1), (8, 1), (64, 64), (800, 800)])
@pytest.mark.parametrize("batch", [1, 16, 80])
def test_a_chunk_workspace_serves_every_smaller_call(n_q, n_kv, batch):
    """As make_chunk_workspace promises: never less for more rows or a wider bound, around 32 query rows (where tiles that share rows
    begin), around tiles of 128 and around the most parts."""
    cfg = B.make_config(batch, n_q, n_kv, 4096)
    rep = n_q // n_kv
    near = {x // rep + d for x in (0, 32, 128, 48 * 128) for d in (-1, 0, 1, 2)}
    ns = sorted({n for n in near | {1, 2, batch, batch + 1, 100, 1000, 5000, 1 << 17, 1 << 24} if 0 <= n <= 1 << 24})
    size = {(n, m): B.chunk_workspace_bytes(cfg, n, m) for n in ns for m in ns}
    for n0, n1 in zip(ns, ns[1:]):
        for m in ns:
            assert 0 < size[n0, m] <= size[n1, m], (n0, n1, m)
            assert size[m, n0] <= size[m, n1], (m, n0, n1)
