"""Operators of a drafted step from their definitions (test infrastructure only): a host's page
allocator, norms of heads with rotary positions and their gradients, attention under bit masks,
and the move of accepted tokens.  Floating point is float64.
"""
from __future__ import annotations

import numpy as np

from oracle import rotary

PAGE = 16


def kv_map(prior, new, held, table, free, num_free, rows, depths=None):
    """Request by request.  free: the stack's whole buffer.  Returns a dict of the call's outputs."""
    table, free = np.array(table, np.int64), np.array(free, np.int64)
    B, columns = table.shape
    prior, new, held = (np.asarray(x, np.int64) for x in (prior, new, held))
    stack = free[:min(max(int(num_free), 0), len(free))].tolist()
    want = -(-(prior + new) // PAGE)
    valid = (prior >= 0) & (new >= 0) & (held >= 0) & (held <= columns) & (want <= columns)
    for b in range(B):
        if valid[b]:
            stack += table[b, want[b]:held[b]].tolist()
    stack = stack[:len(free)]
    free[:len(stack)] = stack
    held_out, refused = held.copy(), np.zeros(B, np.int64)
    starts = np.zeros(B + 1, np.int64)
    slots, positions = np.full(rows, -1, np.int64), np.zeros(rows, np.int64)
    asked, top, total = 0, len(stack), 0
    for b in range(B):
        need = max(0, int(want[b] - held[b])) if valid[b] else 0
        asked += need
        refused[b] = not valid[b] or (need > 0 and asked > top)
        if not refused[b]:
            for j in range(held[b], want[b]):
                table[b, j] = stack.pop()
            held_out[b] = want[b]
        for i in range(max(0, int(new[b]))):
            r, token = total + i, int(prior[b]) + i
            if r >= rows:
                break
            if not refused[b]:
                slots[r] = table[b, token // PAGE] * PAGE + token % PAGE
            positions[r] = np.int64(token if depths is None else prior[b] + depths[r]).astype(np.int32)
        total += max(0, int(new[b]))
        starts[b + 1] = min(total, rows)
    return dict(table=table, free=free, held=held_out, num_free=len(stack), refused=refused,
                starts=starts, slots=slots, positions=positions)


def norm_turn(x, weight, eps, positions, theta, **turn):
    """(y, n, r): x [rows, heads, D] normalised, weighted and turned; the normalised heads; 1 / norm."""
    x, weight = np.asarray(x, np.float64), np.asarray(weight, np.float64)
    r = 1.0 / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + float(np.float32(eps)))
    n = x * r
    return rotary.turn(n * weight, positions, theta, **turn), n, r


def norm_turn_grad(x, weight, eps, positions, theta, dy, **turn):
    """(dx, dweight, terms): the gradients, and the sizes of the terms that each adds up."""
    weight = np.asarray(weight, np.float64)
    _, n, r = norm_turn(x, weight, eps, positions, theta, **turn)
    du = rotary.turn(dy, positions, theta, backward=True, **turn)
    dn = du * weight
    along = np.mean(dn * n, axis=-1, keepdims=True)
    dx = r * (dn - n * along)
    size = rotary.partner_size(dy, theta, turn.get("interleaved", False))
    size = np.where(size > 0, size, np.abs(dy)) * turn.get("amplitude", 1.0)
    terms_x = r * (size * np.abs(weight) + np.abs(n) * np.mean(size * np.abs(weight) * np.abs(n), -1,
                                                               keepdims=True))
    return dx, (du * n).sum(axis=(0, 1)), (terms_x, (size * np.abs(n)).sum(axis=(0, 1)))


def tree_attention(q, keys, values, prior, seen, scale):
    """One request: q [N, Hq, D], keys and values [tokens, Hkv, D], seen [N, N] truth values.
    Returns (out, lse, sizes): sizes[n, h, d] = sum of p |v| over what the row sees, and the
    largest scale * sum |q k| of a row."""
    q, keys, values = (np.asarray(x, np.float64) for x in (q, keys, values))
    N, Hq, D = q.shape
    G = Hq // keys.shape[1]
    out, lse = np.zeros((N, Hq, D)), np.full((N, Hq), -np.inf)
    size, score = np.zeros((N, Hq, D)), np.zeros((N, Hq))
    for i in range(N):
        at = np.concatenate([np.arange(prior), prior + np.flatnonzero(seen[i][:len(keys) - prior])])
        if len(at) == 0:
            continue
        for h in range(Hq):
            k, v = keys[at, h // G], values[at, h // G]
            with np.errstate(invalid="ignore", over="ignore"):
                z = float(np.float32(scale)) * (k @ q[i, h])
                m = z.max()
                p = np.exp(z - m)
                out[i, h] = p @ v / p.sum()
                lse[i, h] = m + np.log(p.sum())
                size[i, h] = p @ np.abs(v) / p.sum()
                score[i, h] = float(np.float32(scale)) * (np.abs(k) @ np.abs(q[i, h])).max()
    return out, lse, size, score


def accept(tokens, prior, accepted, count):
    """tokens [n, ...] of one request's cache after the move."""
    out = np.array(tokens)
    for i in range(count):
        if accepted[i] > i:
            out[prior + i] = tokens[prior + accepted[i]]
    return out
