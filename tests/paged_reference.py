"""Plain definitions of the operators on paged requests, in 64 bits and one element after the other where that is affordable.
Nothing here is shared with the library or with perf/operators.py."""
import math

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def half_step(dtype):
    """A rounding's largest relative error: eps / 2."""
    return {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}[dtype]


# ---- block tables -------------------------------------------------------------------------------------------------

def plan(cached, new, owned, table, free_ids, free_count, rows, block_size, n_blocks):
    """The books kept request by request.  Returns a dict of the outputs (lists and arrays)."""
    b, max_blocks = len(cached), table.shape[1]
    table, free_ids, owned = table.copy(), free_ids.copy(), list(owned)
    free = [int(x) for x in free_ids[:free_count]]
    start = list(owned)
    for i in range(b):
        if cached[i] < 0:
            for j in range(owned[i]):
                free.append(int(table[i, j]))
                free_ids[len(free) - 1] = table[i, j]
            owned[i] = 0
    seq, cu, cu_seq, refused, ends = [], [0], [0], False, 0
    for i in range(b):
        ends += max(new[i], 0)
        cu.append(min(ends, rows))
        total = cached[i] + new[i]
        ok = cached[i] >= 0 and new[i] >= 0 and total <= max_blocks * block_size and ends <= rows
        if ok:
            need = max(0, -(-total // block_size) - start[i])
            if need and (refused or need > len(free)):
                refused, ok = True, False
            else:
                for j in range(need):
                    table[i, start[i] + j] = free.pop()
                owned[i] = start[i] + need
        seq.append(total if ok else -1)
        cu_seq.append(cu_seq[-1] + (total if ok else 0))
    slot, pos = np.full(rows, -1, np.int64), np.full(rows, -1, np.int64)
    for i in range(b):
        if seq[i] < 0:
            continue
        for r in range(cu[i], cu[i + 1]):
            p = cached[i] + r - cu[i]
            pos[r] = p
            block = table[i, p // block_size]
            if 0 <= block < n_blocks:
                slot[r] = block * block_size + p % block_size
    return dict(seq_len=seq, cu_rows=cu, cu_seq=cu_seq, owned=owned, free_count=len(free), table=table, free_ids=free_ids, slot=slot,
                position=pos)


# ---- rotary positions -----------------------------------------------------------------------------------------------

def frequencies(n, base, scaling="none", factor=1.0, original=0, fast=32.0, slow=1.0, low=1.0, high=4.0):
    """Radians per position of every pair and the factor on cos and sin, pair by pair."""
    if scaling == "base" and n > 2:
        base = base * factor ** (n / (n - 2))
    out = []
    for i in range(n // 2):
        f = base ** (-2.0 * i / n)
        turns = original * f / (2 * math.pi)
        if scaling == "linear":
            f /= factor
        elif scaling == "parts":
            def index(rotations):
                return n * math.log(original / (rotations * 2 * math.pi)) / (2 * math.log(base))
            lo, hi = max(0, math.floor(index(fast))), min(n - 1, math.ceil(index(slow)))
            ramp = min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
            f = f * (1 - ramp) + f / factor * ramp
        elif scaling == "bands":
            keep = min(1.0, max(0.0, (turns - low) / (high - low)))
            f = f * keep + f / factor * (1 - keep)
        out.append(f)
    return np.array(out), (0.1 * math.log(factor) + 1 if scaling == "parts" else 1.0)


def rope(x, position, freq, size, layout, inverse):
    """x [rows, heads, head_dim] float64."""
    n, y = 2 * len(freq), x.astype(np.float64).copy()
    angle = position.astype(np.float64)[:, None] * freq
    turn = size * np.exp((-1j if inverse else 1j) * angle)[:, None, :]
    z = (x[..., :n // 2] + 1j * x[..., n // 2:n] if layout == "half" else x[..., 0:n:2] + 1j * x[..., 1:n:2]) * turn
    if layout == "half":
        y[..., :n // 2], y[..., n // 2:n] = z.real, z.imag
    else:
        y[..., 0:n:2], y[..., 1:n:2] = z.real, z.imag
    return y


# ---- the cache ------------------------------------------------------------------------------------------------------

def held_plain(x):
    """What rows [..., head_dim] (any float) are held as, value by value: float64."""
    g = np.asarray(x, np.float64).reshape(-1, 32)
    out = np.empty_like(g)
    for i, row in enumerate(g):
        if not np.all(np.isfinite(row)):
            out[i] = np.nan
            continue
        most = np.abs(row).max()
        e = -126
        if most > 0:
            m, p = math.frexp(most / 6)                     # most / 6 = m * 2^p, 1/2 <= m < 1
            e = max(-126, p - 1 if m == 0.5 else p)
        unit = math.ldexp(1.0, e)
        for j, v in enumerate(row):
            d = np.abs(abs(v) / unit - LEVELS)
            near = np.flatnonzero(d == d.min())
            code = near[0] if len(near) == 1 or near[0] % 2 == 0 else near[1]      # the even code among equals
            out[i, j] = math.copysign(LEVELS[code] * unit, v)
    return out.reshape(np.shape(x))


def held(x):
    """The same for many rows at once."""
    g = np.asarray(x, np.float64).reshape(-1, 32)
    bad = ~np.isfinite(g).all(1)
    g = np.where(bad[:, None], 0.0, g)
    m, p = np.frexp(np.abs(g).max(1) / 6)
    e = np.maximum(np.where(m == 0.5, p - 1, p), -126)
    e[np.abs(g).max(1) == 0] = -126
    unit = np.ldexp(1.0, e)[:, None]
    even = np.argsort(np.arange(8) % 2, kind="stable")        # even codes first: argmin takes the first of equals
    out = np.empty_like(g)
    for i in range(0, len(g), 4096):
        d = np.abs(np.abs(g[i:i + 4096, :, None]) / unit[i:i + 4096, :, None] - LEVELS[even])
        out[i:i + 4096] = np.copysign(LEVELS[even][d.argmin(-1)] * unit[i:i + 4096], g[i:i + 4096])
    out[bad] = np.nan
    return out.reshape(np.shape(x))


def attention(q, k, v, seen, scale):
    """One request: q [n, heads, d], k and v [t, kv_heads, d] float64, seen[i] tokens visible to row i.  Returns out, lse, the
    weighted mean magnitude of the values (what a relative error of the probabilities multiplies), the sum of magnitudes
    of visible values over the largest weight's sum, and the largest sum of magnitudes of a visible score's products."""
    n, heads, d = q.shape
    group = heads // k.shape[1]
    out, mean, flat = np.zeros((n, heads, d)), np.zeros((n, heads, d)), np.zeros((n, heads, d))
    lse, size = np.full((n, heads), -np.inf), np.zeros((n, heads))
    for i in range(n):
        t = int(min(max(seen[i], 0), k.shape[0]))
        if t == 0:
            continue
        for h in range(heads):
            kk, vv = k[:t, h // group], v[:t, h // group]
            with np.errstate(invalid="ignore"):
                s = scale * (kk @ q[i, h])
                m = s.max() if not np.isnan(s).any() else np.nan
                w = np.exp(s - m)
                total = w.sum()
                out[i, h] = w @ vv / total
                mean[i, h] = w @ np.abs(vv) / total
                flat[i, h] = np.abs(vv).sum(0) / total
                lse[i, h] = m + np.log(total)
                size[i, h] = abs(scale) * (np.abs(kk) @ np.abs(q[i, h])).max()
    return out, lse, mean, flat, size
