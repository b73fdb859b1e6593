"""CPU oracle for attention over a paged cache, in 64 bits, one row at a time.

TEST INFRASTRUCTURE ONLY.  The product path never calls it and shares no code
with it.

  cache   pool[page][plane][slot][head][dim] of one layer (slot-major), floats
  token at position p of request r, query head h, KV head g = h // (Hq / Hkv):
    V   = { j <= p : W == 0 or j > p - W or j < S }, less positions whose table entry is not a page
    x_j = scale * q . key_j
    out = sum_V exp(x_j) value_j / sum_V exp(x_j);  lse = ln sum_V exp(x_j)
  an empty V gives out = 0, lse = -inf.

With two planes plane 0 holds keys and plane 1 values, with one plane the
value is the key row's first `value_dim` elements.
"""
from __future__ import annotations

import numpy as np


def visible(position: int, window: int, sinks: int) -> list:
    return [j for j in range(position + 1) if window == 0 or j > position - window or j < sinks]


def attend_row(pool, table, position, q, kv_head, scale, value_dim, window=0, sinks=0):
    """(out [value_dim], lse, spread [value_dim], size) of one query row.

    spread = sum softmax |value| and size = max_j scale * sum |q_d key_jd| are
    what the error bounds of a kernel are made of."""
    num_pages, planes, page_size = pool.shape[:3]
    rows = []
    for j in visible(position, window, sinks):
        e = int(table[j // page_size])
        if 0 <= e < num_pages:
            rows.append((e, j % page_size))
    if not rows:
        return np.zeros(value_dim), -np.inf, np.zeros(value_dim), 0.0
    e, s = (np.array(c) for c in zip(*rows))
    keys = pool[e, 0, s, kv_head]
    values = pool[e, planes - 1, s, kv_head][:, :value_dim]
    x = scale * (keys @ q)
    top = x.max()
    p = np.exp(x - top)
    total = p.sum()
    p /= total
    return p @ values, top + np.log(total), p @ np.abs(values), float((scale * (np.abs(keys) @ np.abs(q))).max())


def attend(pool, tables, seq_lens, q_starts, q, kv_heads, scale, value_dim, window=0, sinks=0, head_begin=0, only=None):
    """Every row of q [tokens][heads][dim] that belongs to a request (of the
    tokens in `only`, if given): a dict keyed by (token, head) of attend_row's
    answers."""
    heads = q.shape[1]
    got = {}
    for r, n in enumerate(seq_lens):
        first, last = int(q_starts[r]), int(q_starts[r + 1])
        for t in range(first, last):
            if only is not None and t not in only:
                continue
            position = int(n) - (last - t)
            for h in range(heads):
                got[t, h] = attend_row(pool, tables[r], position, q[t, h], head_begin + h // (heads // kv_heads), scale,
                                       value_dim, window, sinks)
    return got
