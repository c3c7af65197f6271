"""The operators that bring prompts and chunks of new tokens into the cache, case by case, in two forms: as calls of this
library, and as plain torch operations in 32 bits.

A case is a dict of plain values.  `kind` names the operator:
  prefill  causal attention over whole prompts that lie packed one after the other (grouped heads, unequal lengths)
  chunk    attention of each sequence's new tokens over its cache rows, contiguous or paged; the new rows are in the cache
  append   a chunk's K / V rows written into the cache and the 1-bit copy of the keys extended over them
  table    block table, packed offsets and slot map from the lengths before and after a step
Lengths: `ctx` tokens in the cache before the call and `new` tokens in it, the same for every sequence, or spread over
[ctx_lo, ctx] and [new_lo, new] where the lower bound is smaller.
"""
import math

import numpy as np
import torch

own = False  # whether run() makes the library's calls

D = 128
_BASE = dict(kind="prefill", batch=1, n_q_heads=8, n_kv_heads=8, ctx_lo=0, ctx=0, new_lo=0, new=1, dtype="f16", group=32,
             block_tokens=0, fused_qkv=False, padding=0, done=0)


def _case(name, **kw):
    c = dict(_BASE, name=name, **kw)
    c["ctx_lo"] = kw.get("ctx_lo", c["ctx"])
    c["new_lo"] = kw.get("new_lo", c["new"])
    return c


def listed():
    return [
        # one short question: launches and latency
        _case("prefill-100", new=100),
        # one ordinary prompt of a grouped-query layer
        _case("prefill-4k-gqa", n_q_heads=32, new=4096, dtype="bf16"),
        # a long document through a 32-head layer: the largest
        _case("prefill-16k", n_q_heads=32, n_kv_heads=32, new=16384),
        # a batch of unequal prompts packed by a server, views of one fused q/k/v product, padded to a fixed size
        _case("prefill-ragged", batch=16, n_q_heads=32, new_lo=30, new=2001, dtype="bf16", fused_qkv=True, padding=77),
        # one token each of 16 long conversations, paged rows
        _case("chunk-1-ragged", kind="chunk", batch=16, n_q_heads=32, ctx_lo=8192, ctx=65536, dtype="bf16", block_tokens=64),
        # a chunk of a long prompt between decode steps: 512 tokens behind 32k
        _case("chunk-512-32k", kind="chunk", n_q_heads=32, ctx=32768, new=512, dtype="bf16", block_tokens=128),
        # five drafted tokens per sequence to be verified, multi-head, contiguous rows
        _case("chunk-5-4k", kind="chunk", batch=8, n_q_heads=32, n_kv_heads=32, ctx_lo=3000, ctx=4100, new=5),
        # single tokens and pieces of prompts in one batch
        _case("chunk-mixed", kind="chunk", batch=8, n_q_heads=24, ctx_lo=0, ctx=12000, new_lo=1, new=500, dtype="bf16",
              block_tokens=64),
        # a whole prompt's keys and values into an empty cache
        _case("append-32k", kind="append", n_q_heads=32, n_kv_heads=32, new=32768),
        # chunks of unequal sequences, group and block boundaries anywhere, larger quantization groups
        _case("append-ragged-g128", kind="append", batch=12, n_q_heads=32, ctx_lo=100, ctx=9000, new_lo=20, new=700,
              dtype="bf16", group=128, block_tokens=128, fused_qkv=True),
        # the table of a decode step: every sequence grows by a token, a few have ended
        _case("table-step", kind="table", batch=64, ctx_lo=100, ctx=8000, new=1, done=3, block_tokens=64),
        # a batch of prompts admitted at once, beside sequences that end
        _case("table-admit", kind="table", batch=256, ctx_lo=0, ctx=4000, new_lo=1, new=6000, done=40, block_tokens=64),
    ]


def draw(rng):
    between = lambda lo, hi: int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999))))  # noqa: E731
    kind = rng.choice(["prefill"] * 3 + ["chunk"] * 4 + ["append"] * 2 + ["table"])
    n_q, n_kv = rng.choice([(8, 8), (16, 8), (24, 8), (32, 8), (64, 8), (28, 4), (32, 32), (5, 1)])
    c = dict(_BASE, kind=kind, n_q_heads=n_q, n_kv_heads=n_kv, dtype=rng.choice(["f16", "bf16"]), batch=between(1, 16))
    c["group"] = rng.choice([32, 32, 64, 128])
    if kind == "prefill":
        c["new"] = between(1, 8000)
        c["new_lo"] = max(1, int(c["new"] * rng.choice([1.0, 0.5, 0.05])))
    elif kind == "table":
        c["batch"] = between(1, 256)
        c["ctx"], c["new"] = between(1, 8000), between(1, 6000)
        c["ctx_lo"], c["new_lo"] = rng.choice([0, c["ctx"] // 2]), 1
        c["done"] = rng.randrange(0, c["batch"] // 2 + 1)
    else:
        c["ctx"] = between(1, 65536) if kind == "chunk" else between(1, 16000)
        c["ctx_lo"] = int(c["ctx"] * rng.choice([1.0, 0.5, 0.1]))
        c["new"] = rng.choice([1, between(1, 16), between(1, 1024)])
        c["new_lo"] = max(1, int(c["new"] * rng.choice([1.0, 0.3])))
    if kind in ("chunk", "append"):
        c["block_tokens"] = rng.choice([0, max(64, c["group"]), max(64, c["group"]), 256])
    if kind == "table":
        c["block_tokens"] = rng.choice([64, 128, 256])
        c["group"] = 32
    if kind in ("prefill", "append"):
        c["fused_qkv"] = rng.random() < 0.5
    if kind in ("prefill", "chunk"):
        c["padding"] = rng.choice([0, 0, rng.randrange(1, 100)])
        # the plain form's square of scores bounds the batch
        while c["batch"] * c["n_q_heads"] * c["new"] * (c["ctx"] + c["new"]) > 3e9 and c["batch"] > 1:
            c["batch"] //= 2
        while c["batch"] * c["n_q_heads"] * c["new"] * (c["ctx"] + c["new"]) > 3e9:
            c["new"] = max(1, c["new"] // 2)
            c["new_lo"] = min(c["new_lo"], c["new"])
    while c["kind"] != "table" and c["batch"] > 1 and c["batch"] * n_kv * (c["ctx"] + c["new"]) > 2e6:
        c["batch"] //= 2
    return c


def _lens(case):
    """Lengths before the call and new tokens of every sequence: part of the case, not of its inputs."""
    rng = np.random.default_rng([case["batch"], case["ctx"], case["new"]])
    old = rng.integers(case["ctx_lo"], case["ctx"] + 1, size=case["batch"])
    new = rng.integers(case["new_lo"], case["new"] + 1, size=case["batch"])
    old[-1], new[-1] = case["ctx"], case["new"]
    if case["kind"] == "table":  # sequences that end give all their blocks back
        gone = rng.permutation(case["batch"])[: case["done"]]
        new[gone] = -old[gone]
    return old.astype(np.int64), new.astype(np.int64)


def _capacity(case):
    gran = max(64, case["group"], case["block_tokens"])
    return -(-(case["ctx"] + case["new"]) // gran) * gran


def work(case):
    old, new = _lens(case)
    kind, n_q, n_kv = case["kind"], case["n_q_heads"], case["n_kv_heads"]
    n = int(new.sum())
    if kind == "table":
        bt = case["block_tokens"]
        moved = int(np.abs(-(-(old + new) // bt) - -(-old // bt)).sum())
        slots = int(np.maximum(new, 0).sum())
        # lengths, moved blocks (from one list to the other), offsets, slots
        return {"bytes": 12 * case["batch"] + 8 * moved + 4 * slots, "flops": 4 * case["batch"] + slots}
    if kind == "append":
        packed = 16 + 512 // case["group"]
        head = int((old % case["group"]).sum())  # rows of the groups that the chunks continue
        return {"bytes": int(n_kv * (n * (8 * D + packed) + head * 2 * D)), "flops": int(n_kv * (n + head) * 3 * D)}
    rows = int((old + new).sum())
    pairs = int((new * old + new * (new + 1) // 2).sum())
    return {"bytes": 2 * D * (2 * n_q * n + 2 * n_kv * rows), "flops": 4 * D * n_q * pairs}


# ---- inputs -----------------------------------------------------------------------------------------------------------


def _i32(a):
    return torch.as_tensor(np.asarray(a, np.int32), device="cuda")


def _keys(gen, shape, dtype, heads_dim):
    """Keys with a few channels eight times the others, as in trained models."""
    scale = torch.ones((shape[heads_dim], D), device="cuda")
    scale.scatter_(1, torch.rand(scale.shape, generator=gen, device="cuda").topk(4, dim=1).indices, 8.0)
    view = [1] * len(shape)
    view[heads_dim], view[-1] = shape[heads_dim], D
    return (torch.randn(shape, generator=gen, device="cuda") * scale.view(view)).to(dtype)


def prepare(case, seed):
    """A program between two steps: its cache (contiguous, or a pool of blocks with a table), the new tokens' rows as its
    projections left them, lengths and offsets on the GPU, outputs and the workspace it keeps."""
    kind, b, n_q, n_kv = case["kind"], case["batch"], case["n_q_heads"], case["n_kv_heads"]
    old, new = _lens(case)
    cap, bt = _capacity(case), case["block_tokens"]
    dtype = torch.float16 if case["dtype"] == "f16" else torch.bfloat16
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": case, "cap": cap}
    if kind == "table":
        held = -(-old // bt)
        n_pool = int(np.maximum(held, -(-(old + new) // bt)).sum()) + 500
        perm = torch.randperm(n_pool, generator=gen, device="cuda").to(torch.int32)
        s["table"] = torch.zeros((b, cap // bt), dtype=torch.int32, device="cuda")
        entries = torch.arange(cap // bt, device="cuda")[None, :] < _i32(held)[:, None]
        s["table"][entries] = perm[: int(held.sum())]
        n_free = n_pool - int(held.sum())
        s["free"] = torch.cat([perm[int(held.sum()):], torch.zeros(n_pool - n_free, dtype=torch.int32, device="cuda")])
        s["n_free"], s["n_free_out"] = _i32([n_free]), _i32([0])
        s["old_lens"], s["new_lens"] = _i32(old), _i32(old + new)
        s["starts"] = torch.zeros(b + 1, dtype=torch.int32, device="cuda")
        s["slots"] = torch.zeros(max(1, int(np.maximum(new, 0).sum())), dtype=torch.int32, device="cuda")
    else:
        n = int(new.sum())
        rows = n + case["padding"]
        starts = np.concatenate([[0], np.cumsum(new)])
        s["starts"], s["seq_lens"], s["max_new"], s["n"] = _i32(starts), _i32(old), int(new.max()), n
        qkv = torch.empty((rows, n_q + 2 * n_kv, D), dtype=dtype, device="cuda")
        qkv[:, :n_q] = torch.randn((rows, n_q, D), generator=gen, device="cuda") * 0.7
        qkv[:, n_q:n_q + n_kv] = _keys(gen, (rows, n_kv, D), dtype, 1)
        qkv[:, n_q + n_kv:] = torch.randn((rows, n_kv, D), generator=gen, device="cuda") + 0.1
        q, k, v = qkv[:, :n_q], qkv[:, n_q:n_q + n_kv], qkv[:, n_q + n_kv:]
        s["q"], s["k"], s["v"] = (q, k, v) if case["fused_qkv"] else (q.contiguous(), k.contiguous(), v.contiguous())
        s["out"] = torch.zeros((rows, n_q, D), dtype=dtype, device="cuda")
    if kind in ("chunk", "append"):
        if bt:
            n_pool = b * (cap // bt) + 7
            s["table"] = torch.randperm(n_pool, generator=gen, device="cuda")[: b * (cap // bt)].to(torch.int32).view(b, -1)
            shape = (n_pool, n_kv, bt, D)
        else:
            s["table"] = None
            shape = (b * n_kv, cap, D)
        hd = 1 if bt else 0
        s["K"], s["V"] = _keys(gen, shape, dtype, hd), (torch.randn(shape, generator=gen, device="cuda") + 0.1).to(dtype)
        s["kbits"] = torch.zeros((b * n_kv, cap, 4), dtype=torch.int32, device="cuda")
        s["kmeta"] = torch.zeros((b * n_kv, cap // case["group"], D), dtype=torch.int32, device="cuda")
        s["kabsmax"] = torch.zeros((b * n_kv, D), dtype=torch.float32, device="cuda")
        if kind == "append":  # what the cache holds already has its 1-bit copy
            _quantize(s, torch.zeros_like(s["seq_lens"]), s["seq_lens"], np.zeros_like(old), old)
        else:
            _write_rows(s)
    if own:
        from paper_2508_08256_amd import binding as B

        code = B.F16 if case["dtype"] == "f16" else B.BF16
        s["cfg"] = B.make_config(b, n_q, n_kv, cap, code, group_size=case["group"])
        if kind in ("chunk", "append"):
            s["cache"] = B.DeviceCache(s["cfg"], s["K"], s["V"], s["seq_lens"], s["table"])
            for name in ("kbits", "kmeta", "kabsmax"):
                getattr(s["cache"], name).copy_(s[name].view(-1))
                s[name] = getattr(s["cache"], name).view(s[name].shape)
        if kind == "chunk":
            s["ws"] = B.make_chunk_workspace(s["cfg"], s["q"].shape[0], s["max_new"])
    return s


# ---- the plain forms --------------------------------------------------------------------------------------------------


def _tokens(s):
    """Sequence and position in it of every packed new token."""
    t = torch.arange(s["n"], device="cuda")
    b = torch.searchsorted(s["starts"][1:].long(), t, right=True)
    return b, s["seq_lens"].long()[b] + t - s["starts"].long()[b]


def _write_rows(s):
    case = s["case"]
    b, pos = _tokens(s)
    h = torch.arange(case["n_kv_heads"], device="cuda")[None, :]
    if s["table"] is None:
        at = (b[:, None] * case["n_kv_heads"] + h, pos[:, None].expand(-1, case["n_kv_heads"]))
    else:
        bt = case["block_tokens"]
        at = (s["table"].long()[b, pos // bt][:, None], h, (pos % bt)[:, None])
    s["K"][at] = s["k"][: s["n"]]
    s["V"][at] = s["v"][: s["n"]]


def _quantize(s, first, last, first_host, last_host):
    """The 1-bit copy of every block of max(g, 64) tokens that holds one of the tokens [first, last) of its sequence."""
    case, g = s["case"], s["case"]["group"]
    n_kv, span = case["n_kv_heads"], max(s["case"]["group"], 64)
    total = int(np.where(last_host > first_host, -(-last_host // span) - first_host // span, 0).sum())
    first, last = first.long(), last.long()
    count = torch.where(last > first, (last + span - 1) // span - first // span, 0)
    b = torch.repeat_interleave(torch.arange(case["batch"], device="cuda"), count, output_size=total)
    block = torch.arange(total, device="cuda") - (count.cumsum(0) - count)[b] + (first // span)[b]
    pos = block[:, None] * span + torch.arange(span, device="cuda")
    h = torch.arange(n_kv, device="cuda")[None, :, None]
    if s["table"] is None:
        at = (b[:, None, None] * n_kv + h, pos[:, None, :])
    else:
        bt = case["block_tokens"]
        at = (s["table"].long()[b[:, None], pos // bt][:, None, :], h, (pos % bt)[:, None, :])
    dtype = s["K"].dtype
    x = s["K"][at].float().view(total, n_kv, span // g, g, D)
    there = (pos < last[b][:, None]).view(total, 1, span // g, g, 1)
    some = there.any(dim=3)
    z = torch.where(some, torch.where(there, x, math.inf).amin(dim=3), 0.0) + 0.0
    top = torch.where(some, torch.where(there, x, -math.inf).amax(dim=3), 0.0)
    scale = (top - z + 0.0).clamp(max=torch.finfo(dtype).max).to(dtype)
    d = x - z[:, :, :, None]
    bit = ((d + d >= scale.float()[:, :, :, None]) & there).view(total, n_kv, span, 2, 32, 2)
    # word 2 o + u of a token: channels 64 u + 2 i + o, i = 0..31
    words = (bit.permute(0, 1, 2, 5, 3, 4).long() << torch.arange(32, device="cuda")).sum(dim=-1).view(total, n_kv, span, 4)
    raw = lambda t: t.view(torch.int16).long() & 0xFFFF  # noqa: E731
    meta = raw(scale) | raw(z.to(dtype)) << 16
    unit = b[:, None] * n_kv + torch.arange(n_kv, device="cuda")
    s["kbits"].view(case["batch"] * n_kv, -1, span, 4)[unit, block[:, None]] = words.to(torch.int32)
    s["kmeta"].view(case["batch"] * n_kv, -1, span // g, D)[unit, block[:, None]] = meta.to(torch.int32)
    most = torch.maximum(z.abs(), (z + scale.float()).abs()).amax(dim=2)
    s["kabsmax"].index_reduce_(0, unit.view(-1), most.view(-1, D), "amax")


def _attention(s, K, V, first):
    """K, V: [batch][kv heads][rows][D], sequence b's new token i at row first[b] + i."""
    case = s["case"]
    n_kv, rep, batch, width = case["n_kv_heads"], case["n_q_heads"] // case["n_kv_heads"], case["batch"], s["max_new"]
    i = torch.arange(width, device="cuda")
    begin, end = s["starts"].long()[:-1], s["starts"].long()[1:]
    at = torch.minimum(begin[:, None] + i, (end - 1).clamp(min=0)[:, None])
    q = s["q"][at].float().view(batch, width, n_kv, rep, D).permute(0, 2, 3, 1, 4).reshape(batch, n_kv, rep * width, D)
    p = (q * D ** -0.5) @ K.float().transpose(2, 3)
    allowed = torch.arange(K.shape[2], device="cuda") <= (first.long()[:, None] + i)[:, :, None]
    p = p.view(batch, n_kv, rep, width, -1).masked_fill_(~allowed[:, None, None], -math.inf)
    p = p.sub_(p.amax(dim=-1, keepdim=True)).exp_()
    total = p.sum(dim=-1, keepdim=True)
    o = (p.view(batch, n_kv, rep * width, -1) @ V.float()).view(batch, n_kv, rep, width, D) / total
    o = o.permute(0, 3, 1, 2, 4).reshape(batch, width, n_kv * rep, D).to(s["out"].dtype)
    b = torch.searchsorted(end, torch.arange(s["n"], device="cuda"), right=True)
    s["out"][: s["n"]] = o[b, torch.arange(s["n"], device="cuda") - begin[b]]
    return s["out"]


def _plain_prefill(s):
    at = torch.minimum(s["starts"].long()[:-1, None] + torch.arange(s["max_new"], device="cuda"),
                       (s["starts"].long()[1:] - 1).clamp(min=0)[:, None])
    return _attention(s, s["k"][at].transpose(1, 2), s["v"][at].transpose(1, 2), torch.zeros_like(s["seq_lens"]))


def _plain_chunk(s):
    case = s["case"]
    if s["table"] is None:
        shape = (case["batch"], case["n_kv_heads"], -1, D)
        return _attention(s, s["K"].view(shape), s["V"].view(shape), s["seq_lens"])
    rows = lambda pool: pool[s["table"].long()].transpose(1, 2).reshape(case["batch"], case["n_kv_heads"], -1, D)  # noqa: E731
    return _attention(s, rows(s["K"]), rows(s["V"]), s["seq_lens"])


def _plain_append(s):
    old, new = _lens(s["case"])
    _write_rows(s)
    _quantize(s, s["seq_lens"], s["seq_lens"] + (s["starts"][1:] - s["starts"][:-1]), old, old + new)
    return s["K"], s["V"], s["kbits"], s["kmeta"], s["kabsmax"]


def _plain_table(s):
    case, bt, table, free = s["case"], s["case"]["block_tokens"], s["table"], s["free"]
    old, new, n = s["old_lens"].long().clamp(0, s["cap"]), s["new_lens"].long().clamp(0, s["cap"]), s["n_free"].long()
    before = lambda x: x.cumsum(0) - x  # noqa: E731
    held, want = (old + bt - 1) // bt, (new + bt - 1) // bt
    give, take = (held - want).clamp(min=0), (want - held).clamp(min=0)
    left = n + give.sum() - take.sum()
    ok = left >= 0
    e = torch.arange(table.shape[1], device="cuda")[None, :]
    # the blocks given back go on top of the stack of free ones, those taken come from its top
    back = (e >= want[:, None]) & (e < held[:, None])
    spot = torch.where(back, n + before(give)[:, None] + e - want[:, None], free.numel())
    stack = torch.cat([free, free.new_zeros(1)]).scatter_(0, spot.view(-1), table.view(-1))
    taken = ok & (e >= held[:, None]) & (e < want[:, None])
    spot = n + give.sum() - 1 - before(take)[:, None] - (e - held[:, None])
    table.copy_(torch.where(taken, stack[spot.clamp(0, free.numel() - 1)], table))
    p = torch.arange(free.numel(), device="cuda")
    free.copy_(torch.where(ok & (p >= n) & (p < left), stack[:-1], free))
    s["n_free_out"].copy_(left)
    grown = (new - old).clamp(min=0)
    starts = torch.cat([grown.new_zeros(1), grown.cumsum(0)])
    s["starts"].copy_(torch.where(ok, starts, s["starts"].long()))
    t = torch.arange(s["slots"].numel(), device="cuda")
    b = torch.searchsorted(starts[1:], t, right=True).clamp(max=case["batch"] - 1)
    pos = (old[b] + t - starts[b]).clamp(0, s["cap"] - 1)
    slot = table[b, pos // bt].long() * bt + pos % bt
    s["slots"].copy_(torch.where(ok & (t < starts[-1]), slot, s["slots"].long()))
    return table, free, s["n_free_out"], s["starts"], s["slots"]


def run(s):
    kind = s["case"]["kind"]
    if not own:
        return {"prefill": _plain_prefill, "chunk": _plain_chunk, "append": _plain_append, "table": _plain_table}[kind](s)
    from paper_2508_08256_amd import binding as B

    if kind == "prefill":
        B.prefill_attn(s["cfg"], s["q"], s["k"], s["v"], s["starts"], s["max_new"], s["out"])
        return s["out"]
    if kind == "chunk":
        B.chunk_attn(s["cfg"], s["cache"], s["q"], s["starts"], s["max_new"], s["out"], s["ws"])
        return s["out"]
    if kind == "append":
        B.append_chunk(s["cfg"], s["cache"], s["k"], s["v"], s["starts"], s["max_new"])
        return s["K"], s["V"], s["kbits"], s["kmeta"], s["kabsmax"]
    B.block_table(s["cfg"], s["case"]["block_tokens"], s["old_lens"], s["new_lens"], s["table"], s["free"], s["n_free"],
                  s["n_free_out"], s["starts"], s["slots"])
    return s["table"], s["free"], s["n_free_out"], s["starts"], s["slots"]


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------


def exact(case, seed):
    if case["kind"] == "table":
        return None  # whole numbers only
    s = prepare(case, seed)
    old, new = _lens(case)
    n_kv, rep, bt = case["n_kv_heads"], case["n_q_heads"] // case["n_kv_heads"], case["block_tokens"]

    def cache_rows(rows, b, h, n):  # rows 0..n-1 of sequence b, kv head h
        if not bt:
            return rows[b * n_kv + h, :n]
        return torch.cat([rows[int(j), h] for j in s["table"][b, : -(-n // bt)]])[:n] if n else rows[0, h, :0]

    if case["kind"] == "append":
        K, V, at, top = s["K"].double(), s["V"].double(), 0, s["kabsmax"].double()
        for b in range(case["batch"]):
            lo, end = int(old[b]), int(old[b] + new[b])
            while lo < end:  # the rows that lie in one block
                hi = min(end, (lo // bt + 1) * bt) if bt else end
                for whole, part in ((K, s["k"]), (V, s["v"])):
                    x = part[at:at + hi - lo].double().transpose(0, 1)
                    if bt:
                        whole[int(s["table"][b, lo // bt]), :, lo % bt:lo % bt + hi - lo] = x
                    else:
                        whole[b * n_kv:(b + 1) * n_kv, lo:hi] = x
                at, lo = at + hi - lo, hi
            g = case["group"]
            begin = int(old[b]) // g * g
            for h in range(n_kv):  # the largest level of a group: its minimum, or that plus the rounded range
                x = cache_rows(K, b, h, end)[begin:]
                full = (end - begin) // g * g
                for y in (x[:full].view(-1, g, D), x[full:].view(-1, max(1, end - begin - full), D)):
                    if y.numel():
                        lo, rng = y.amin(1), (y.amax(1) - y.amin(1)).to(s["K"].dtype).double()
                        most = torch.maximum(lo.abs(), (lo + rng).abs()).amax(0)
                        top[b * n_kv + h] = torch.maximum(top[b * n_kv + h], most)
        return K, V, None, None, top

    out = s["out"].double()
    at = 0
    for b in range(case["batch"]):
        n = int(new[b])
        first = int(old[b]) if case["kind"] == "chunk" else 0
        for h in range(n_kv):
            if case["kind"] == "chunk":
                k, v = cache_rows(s["K"], b, h, first + n).double(), cache_rows(s["V"], b, h, first + n).double()
            else:
                k, v = s["k"][at:at + n, h].double(), s["v"][at:at + n, h].double()
            for r in range(rep):
                logits = s["q"][at:at + n, h * rep + r].double() @ k.T / math.sqrt(D)
                logits += torch.full_like(logits, -math.inf).triu_(first + 1)
                out[at:at + n, h * rep + r] = torch.softmax(logits, dim=1) @ v
        at += n
    return out
