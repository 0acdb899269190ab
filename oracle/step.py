"""Oracle of the operators of a speculative step that can be called alone.  TEST INFRASTRUCTURE ONLY.

Written from the definitions, in float64, one request and one row at a time:

  tables      need = max(0, ceil((ctx + new) / 16) - held); blocks from the top of the stack, in request order; row i of a
              request stands at position ctx + i, in slot (its block) * 16 + position % 16
  norm, rope  y = x / sqrt(mean(x^2) + eps) * gain; (y_i, y_{i + hd/2}) turned by position * theta^(-2i/hd)
  attention   a row at position p sees key j <= p when j > p - window (window 0: always) or j < sinks
  verify      accept x while u q(x) < p(x); then one token by the inverse of the running sum of max(0, p - q), or of p
"""
from __future__ import annotations

import math

import numpy as np

BS = 16


def build_tables(ctx, new, held, free, count, table, max_rows):
    """Returns (row_start, kv_len, positions, slots, held, count, status, table); status as the library names it."""
    n, stride = table.shape
    table = table.copy()
    none = (np.zeros(n + 1, int), np.zeros(n, int), np.full(max_rows, -1), np.full(max_rows, -1), np.array(held), count)
    if min(min(ctx), min(new), min(held), count) < 0 or count > len(free):
        return none + (-2, table)
    if any(h > stride or -(-(c + m) // BS) > stride for c, m, h in zip(ctx, new, held)) or sum(new) > max_rows:
        return none + (-8, table)
    need = [max(0, -(-(c + m) // BS) - h) for c, m, h in zip(ctx, new, held)]
    if sum(need) > count:
        return none + (-6, table)
    stack = [int(x) for x in free[:count]]
    pos, slots, start = [], [], [0]
    for r in range(n):
        for j in range(need[r]):
            table[r, held[r] + j] = stack.pop()
        for i in range(new[r]):
            p = ctx[r] + i
            block = int(table[r, p // BS])
            pos.append(p)
            slots.append(block * BS + p % BS if 0 <= block < 1 << 27 else -1)
        start.append(start[-1] + new[r])
    pad = [-1] * (max_rows - len(pos))
    return (np.array(start), np.array(ctx) + np.array(new), np.array(pos + pad), np.array(slots + pad),
            np.array(held) + np.array(need), count - sum(need), 0, table)


def norm_rope(x, gain, positions, theta, eps):
    """x [rows, heads, hd].  Also returns the sizes of the two terms of each value, for the bound of its error."""
    x = np.asarray(x, np.float64)
    hd = x.shape[-1]
    if gain is not None:
        x = x / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps) * np.asarray(gain, np.float64)
    i = np.arange(hd // 2)
    angle = np.asarray(positions, np.float64)[:, None] * float(theta) ** (-2.0 * i / hd)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    a, b = x[..., :hd // 2], x[..., hd // 2:]
    size = np.concatenate([abs(a) + abs(b)] * 2, -1)
    return np.concatenate([a * c - b * s, b * c + a * s], -1), size


def visible(p, window, sinks):
    j = np.arange(max(0, p + 1))
    return j[(j > p - window) | (j < sinks)] if window else j


def window_attention(q, keys, values, first, window, sinks):
    """q [rows, Hq, hd] of one request whose first row is at position `first`; keys, values [len, Hkv, hd] of its positions.
    Returns the output, sum_j p_j |v_j|, and the largest sum_d |q_d k_d| / sqrt(hd) of each (row, head)."""
    q, keys, values = (np.asarray(t, np.float64) for t in (q, keys, values))
    rows, Hq, hd = q.shape
    rep = Hq // keys.shape[1]
    out, size, spread = np.zeros_like(q), np.zeros_like(q), np.zeros((rows, Hq))
    for i in range(rows):
        j = visible(first + i, window, sinks)
        if len(j) == 0:
            continue
        for h in range(Hq):
            k, v = keys[j, h // rep], values[j, h // rep]
            s = k @ q[i, h] / math.sqrt(hd)
            p = np.exp(s - s.max())
            p /= p.sum()
            out[i, h], size[i, h] = p @ v, p @ abs(v)
            spread[i, h] = (abs(k) @ abs(q[i, h])).max() / math.sqrt(hd)
    return out, size, spread


def target_probs(logits, temperature):
    """Probabilities of a row, and whether it stands for its largest entry alone."""
    z = np.asarray(logits, np.float64)
    z = np.where(np.isnan(z), -np.inf, z)
    best = int(np.flatnonzero(z == z.max())[0])
    if not (temperature > 0 and np.isfinite(temperature)) or not np.isfinite(z[best]):
        p = np.zeros(len(z))
        p[best] = 1.0
        return p, True
    e = np.exp((z - z[best]) / np.float64(temperature))
    return e / e.sum(), False


def verify_request(logits, drafts, probs, temperature, u_accept, u_pick):
    """logits [k + 1, V], drafts [k], probs [k (or more), V] or None.  Returns (tokens [k + 1], accepted), and how near the closest
    decision was (relative to its threshold), so that a test can tell a wrong token from a tie."""
    k, V = len(drafts), logits.shape[1]
    accepted, near = 0, math.inf
    for i in range(k):
        p, one = target_probs(logits[i], temperature)
        x = int(drafts[i])
        if one:
            ok = 0 <= x < V and p[x] == 1.0
        elif not 0 <= x < V:
            ok = False
        else:
            q = float(probs[i, x]) if probs is not None else 1.0
            ok = float(u_accept[i]) * q < p[x]
            if p[x] > 0:
                near = min(near, abs(float(u_accept[i]) * q / p[x] - 1.0))
        if not ok:
            break
        accepted += 1
    p, one = target_probs(logits[accepted], temperature)
    rest = p
    if accepted < k and not one:
        if probs is not None:
            q = np.asarray(probs[accepted], np.float64)
            rest = np.maximum(0.0, p - np.where(q > 0, q, 0.0))
        else:
            rest = p.copy()
            if 0 <= int(drafts[accepted]) < V:
                rest[int(drafts[accepted])] = 0.0
        if not rest.sum() > 0:
            rest = p
    cum = np.cumsum(rest)
    target = np.float64(np.float32(u_pick)) * cum[-1]
    hit = np.flatnonzero((cum > target) & (rest > 0))
    token = int(hit[0]) if len(hit) else int(np.flatnonzero(rest > 0)[-1])
    if not one and not np.isnan(target):
        near = min(near, float(np.min(abs(cum[rest > 0] - target)) / cum[-1]))
    return np.array(list(map(int, drafts[:accepted])) + [token] + [-1] * (k - accepted)), accepted, near
