"""Plain 64-bit statements of the operators around the paged key/value cache (test infrastructure only): loops over requests,
tokens and heads straight from the definitions, in numpy, sharing nothing with the CUDA path."""
from __future__ import annotations

import math

import numpy as np


def pages_of(tokens: int, page_size: int) -> int:
    return -(-tokens // page_size)


def page_plan(cached, added, page_size, table, free, count, capacity, token_cap):
    """One step of the block tables, request by request.  Returns a dict; `table` and `free` are copies, updated."""
    table, free = np.array(table, copy=True), np.array(free, copy=True)
    cached, added = [int(x) for x in cached], [int(x) for x in added]
    B, width = len(cached), table.shape[1]
    out = dict(slot=[-1] * token_cap, position=[0] * token_cap, request=[-1] * token_cap)

    def give_up(state, tokens=0, taken=0, given=0):
        return dict(out, table=table, free=free, count=count, seq_len=cached, q_start=[0] * (B + 1), info=[state, min(tokens, 2**31 - 1), taken, given])

    if not 0 <= count <= capacity or any(c < 0 or a < -1 or c + max(a, 0) > width * page_size for c, a in zip(cached, added)):
        return give_up(1)
    tokens = sum(a for a in added if a > 0)
    given = sum(pages_of(c, page_size) for c, a in zip(cached, added) if a < 0)
    taken = sum(pages_of(c + a, page_size) - pages_of(c, page_size) for c, a in zip(cached, added) if a >= 0)
    if tokens > token_cap:
        return give_up(2, tokens, taken, given)
    if taken > count + given or count + given - taken > capacity:
        return give_up(3, tokens, taken, given)
    stack = [int(x) for x in free[:count]]
    for b in range(B):
        if added[b] < 0:
            stack += [int(x) for x in table[b, :pages_of(cached[b], page_size)]]
    seq_len, q_start, t = [], [0], 0
    for b in range(B):
        if added[b] < 0:
            seq_len.append(0)
        else:
            for i in range(pages_of(cached[b], page_size), pages_of(cached[b] + added[b], page_size)):
                table[b, i] = stack.pop()
            for i in range(added[b]):
                pos = cached[b] + i
                out["slot"][t] = int(table[b, pos // page_size]) * page_size + pos % page_size
                out["position"][t], out["request"][t] = pos, b
                t += 1
            seq_len.append(cached[b] + added[b])
        q_start.append(t)
    free[count:len(stack)] = stack[count:]
    return dict(out, table=table, free=free, count=len(stack), seq_len=seq_len, q_start=q_start, info=[0, tokens, taken, given])


def _pair_index(rot: int, adjacent: bool):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if adjacent else (i, i + rot // 2)


def rotate(x, position, inv_freq, adjacent: bool, back: bool = False):
    """x [T, H, d] fp64; angles reduced by math.fmod on integers times fp64 frequencies."""
    x = np.array(x, dtype=np.float64, copy=True)
    if inv_freq is None or len(inv_freq) == 0:
        return x
    a, b = _pair_index(2 * len(inv_freq), adjacent)
    angle = np.array([[math.fmod(float(p) * float(f), 2 * math.pi) for f in inv_freq] for p in position])[:, None, :]
    cos, sin = np.cos(angle), np.sin(angle) * (-1 if back else 1)
    xa, xb = x[..., a].copy(), x[..., b].copy()
    x[..., a], x[..., b] = xa * cos - xb * sin, xb * cos + xa * sin
    return x


def norm_rope(x, weight, eps, position, inv_freq, adjacent: bool):
    x = np.asarray(x, dtype=np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
    return rotate(x, position, inv_freq, adjacent)


def norm_rope_grad(dy, x, weight, eps, position, inv_freq, adjacent: bool):
    """(dx, dw); dw is None without a weight."""
    dn = rotate(dy, position, inv_freq, adjacent, back=True)
    if weight is None:
        return dn, None
    x = np.asarray(x, dtype=np.float64)
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    g = dn * weight
    return r * (g - x * r * r * (g * x).mean(-1, keepdims=True)), (dn * x * r).sum((0, 1))


def gather(cache, table_row, length: int, page_size: int, heads_first: bool):
    """[length, kv_heads, d] rows of one request."""
    rows = [cache[int(table_row[j // page_size]), :, j % page_size] if heads_first else cache[int(table_row[j // page_size]), j % page_size] for j in range(length)]
    return np.stack(rows) if rows else np.zeros((0,) + ((cache.shape[1],) if heads_first else (cache.shape[2],)) + (cache.shape[3],))


def decode(q, keys, values, scale: float):
    """One request: q [H, d], keys and values [length, kv_heads, d]; returns o [H, d] and the log-sum-exp [H]."""
    H, d = q.shape
    o, lse = np.zeros((H, d)), np.full(H, -np.inf)
    group = H // keys.shape[1]
    if len(keys):
        for h in range(H):
            s = scale * (keys[:, h // group] @ q[h])
            top = s.max()
            p = np.exp(s - top)
            o[h], lse[h] = p @ values[:, h // group] / p.sum(), top + math.log(p.sum())
    return o, lse
