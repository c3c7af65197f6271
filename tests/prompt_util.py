"""Plain 64-bit references of the calls that take many new tokens per sequence, and the bounds their results are held to."""
import math

import numpy as np
import torch

from paper_2508_08256_amd import binding as B

D = 128


def tdtype(dtype):
    return torch.float16 if dtype == B.F16 else torch.bfloat16


def attention64(q, k, v, first, scale, cap=None):
    """q [n][heads][D], k, v [rows][kv heads][D] (any type): token i attends over rows 0 .. first + i.  Returns the outputs and
    how far a result may be off.
      A weight is off by a factor 1 + u (rounding to the K dtype, u half a step) and by its logit's error: 128 products and 32
    bits of accumulation, at most 132 * 2^-24 of the sum of magnitudes A, once for itself and once for the sum it is divided
    by; the exponent's own rounding, the sum's and exp2's are within 1e-5.  The result is rounded once more."""
    n, heads, _ = q.shape
    rep = heads // k.shape[1]
    u = torch.finfo(q.dtype).eps / 2
    out, tol = torch.zeros(n, heads, D, dtype=torch.float64), torch.zeros(n, heads, D, dtype=torch.float64)
    rows = min(first + n, cap) if cap else first + n
    seen = torch.arange(rows)[None, :] <= first + torch.arange(n)[:, None]
    for h in range(heads):
        qh, kh, vh = q[:, h].double(), k[:rows, h // rep].double(), v[:rows, h // rep].double()
        w = torch.softmax(torch.where(seen, scale * (qh @ kh.T), -math.inf), dim=1)
        out[:, h] = w @ vh
        a = torch.where(seen, abs(scale) * (qh.abs() @ kh.abs().T), 0.0).amax(dim=1)
        tol[:, h] = (u + 2 * 132 * 2.0**-24 * a + 1e-5)[:, None] * (w @ vh.abs()) * 1.01 + u * out[:, h].abs() + 1e-30
        if q.dtype == torch.float16:
            tol[:, h] += 2.0**-24 + 2.0**-32 * vh.abs().sum(dim=0)  # subnormal outputs; weights below 2^-21 of the largest
    return out, tol


def check_attention(got, want, tol, what=""):
    err = (got.double().cpu() - want).abs()
    bad = ~(err <= tol)  # a NaN is bad
    assert not bad.any(), (what, int(bad.sum()), float(err.max()), bad.nonzero()[:3].tolist())


def starts_of(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def block_table_plain(block_tokens, max_ctx, old, new, table, free, n_free):
    """(n_free_out, table, free, starts, slots) of fier_block_table; with a negative n_free_out the rest as it was."""
    table, free = table.copy(), free.copy()
    old, new = np.clip(old, 0, max_ctx), np.clip(new, 0, max_ctx)
    held, want = -(-old // block_tokens), -(-new // block_tokens)
    left = int(n_free - (want - held).sum())
    if left < 0:
        return left, table, free, None, None
    stack = list(free[:n_free])
    for b in range(len(old)):
        stack += list(table[b, want[b]:held[b]])
    for b in range(len(old)):
        for e in range(held[b], want[b]):
            table[b, e] = stack.pop()
    free[n_free:len(stack)] = stack[n_free:]
    starts = starts_of(np.maximum(new - old, 0))
    slots = [table[b, p // block_tokens] * block_tokens + p % block_tokens for b in range(len(old)) for p in range(old[b], new[b])]
    return left, table, free, starts, np.array(slots, np.int32)
