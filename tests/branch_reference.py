"""Plain definitions of the operators on requests that continue others, in 64 bits, one request after the other.  Nothing here is shared with
the library or with perf/more_operators.py."""
import math

import numpy as np


# ---- the next beams --------------------------------------------------------------------------------------------------

def candidates(logits, score, length, done, end_token, power):
    """Of one group: (rank, score, beam, token, length, done) of every continuation, the best first."""
    out = []
    for i, row in enumerate(np.asarray(logits, np.float64)):
        if not score[i] > -math.inf:
            continue
        if done is not None and done[i]:
            n = int(length[i]) if length is not None else 0
            out.append((score[i] * max(n, 1) ** -power, score[i], i, end_token, n, 1))
            continue
        row = np.where(np.isnan(row), -np.inf, row)
        top = row.max()
        if not np.isfinite(top):
            continue
        base = score[i] - top - math.log(np.exp(row - top).sum())
        n = (int(length[i]) if length is not None else 0) + 1
        for v in np.flatnonzero(row > -np.inf):
            s = base + row[v]
            out.append((s * max(n, 1) ** -power, s, i, int(v), n, int(v == end_token)))
    out.sort(key=lambda c: (-c[0], c[2], c[3]))
    return out


# ---- requests that continue others -------------------------------------------------------------------------------------

def reorder(parent, length, owned, table, free_ids, free_count, block_size, trim):
    b, most = table.shape
    free_ids = free_ids.copy()
    free = [int(x) for x in free_ids[:free_count]]
    heirs = {}
    for i in range(b):
        p = parent[i]
        if 0 <= p < b and (p not in heirs or p == i):
            heirs[p] = i
    def blocks(n):
        return max(0, -(-n // block_size))
    kept = {}
    for p in range(b):
        kept[p] = 0 if p not in heirs else min(owned[p], blocks(length[p])) if trim else owned[p]
        for j in range(kept[p], owned[p]):
            free.append(int(table[p, j]))
            free_ids[len(free) - 1] = table[p, j]
    out = np.full((b, most), -1, np.int64)
    len_out, owned_out, source, refused = [-1] * b, [0] * b, [-1] * b, False
    for i in range(b):
        p = parent[i]
        if not 0 <= p < b:
            continue
        if heirs[p] == i:
            out[i, :kept[p]] = table[p, :kept[p]]
            len_out[i], owned_out[i] = length[p], kept[p]
            continue
        if length[p] > most * block_size:
            continue
        need = blocks(length[p])
        if need and (refused or need > len(free)):
            refused = True
            continue
        for j in range(need):
            out[i, j] = free.pop()
        len_out[i], owned_out[i], source[i] = length[p], need, heirs[p] if need else -1
    return dict(len_out=len_out, owned_out=owned_out, table_out=out, copy_from=source, free_ids=free_ids, free_count=len(free))


# ---- weights and eviction ------------------------------------------------------------------------------------------------

def weights(q, k, scale, lse, seen):
    """What the tokens k [t, kv_heads, d] receive from the rows q [n, heads, d], of which row i sees the first seen[i]: [t, kv_heads], the largest
    sum of magnitudes of a score's products, and the largest magnitude of what is subtracted."""
    n, heads, d = q.shape
    out, size = np.zeros(k.shape[:2]), 0.0
    for i in range(n):
        t = int(min(max(seen[i], 0), k.shape[0]))
        for h in range(heads):
            if t == 0 or lse[i, h] == -math.inf:
                continue
            kh = h // (heads // k.shape[1])
            s = scale * (k[:t, kh] @ q[i, h])
            size = max(size, abs(scale) * (np.abs(k[:t, kh]) @ np.abs(q[i, h])).max())
            out[:t, kh] += np.exp(s - lse[i, h])
    return out, size


def cut(weight, keep, recent):
    """Which tokens of one head are left of len(weight), in the order in which they are left."""
    n = len(weight)
    if keep < 0 or keep >= n:
        return list(range(n))
    recent = min(recent, keep)
    first, cand = keep - recent, n - recent
    order = sorted(range(cand), key=lambda t: (-(-math.inf if math.isnan(weight[t]) else weight[t]), math.isnan(weight[t]), t))
    chosen = set(order[:first])
    out = [t if t in chosen else None for t in range(first)]
    behind = iter(sorted(t for t in chosen if t >= first))
    return [next(behind) if t is None else t for t in out] + list(range(cand, n))
