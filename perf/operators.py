"""Serving many requests from one pool of cache blocks: five operators as measurable cases, with their plain forms.

plan     block tables, slots and positions from the requests' lengths (heisd_paged_plan)
rope     rotary positions of packed query and key rows: half and interleaved pairs, part of the head, scaled for long
         contexts, and the transposed rotation that gradients take (heisd_rope)
append   new rows into a cache held in 4 bits, and a request's cached rows back out (heisd_kv4_append, heisd_kv4_gather)
decode   attention of one or a few new rows per request over that cache (heisd_kv4_attention)
prompt   attention of whole prompts or chunks of them, packed, with grouped heads (heisd_prompt_attention)

Where `own` is false run() is elementary torch in 32 bits (angles in 64, whole numbers in 64); where it is true it makes the
library's calls.  Lengths belong to a case, values to a seed.

The cache: a pool of blocks of block_size tokens.  Every group of 32 values of a row is held as 4-bit floats (sign, two bits
of exponent, one of mantissa: 0 .5 1 1.5 2 3 4 6) times a power of two, the smallest for which the largest value is at most
6, kept as its exponent plus 127 in a byte, at least 1; 255 stands for a group with a value that is not finite.  One block of
one head is a cell of bytes: key codes [token][head_dim / 2], value codes [token / 4][16][token % 4][head_dim / 32], key
exponents [token][head_dim / 32], value exponents [token / 4][head_dim / 32][token % 4]; in a byte of codes the low half
comes first.
"""
import math
import random
from types import SimpleNamespace

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
GROUP = 32
HALF_STEPS = (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)             # between neighbouring 4-bit values
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # One episode's draft of seven tokens behind its 276-row prefix: launch latency.
        dict(name="plan_1", kind="plan", batch=1, block=16, cached=276, new=7, ragged=False),
        # A full house: 512 requests, prompts and single tokens mixed, some finished, 64-token blocks.
        dict(name="plan_512", kind="plan", batch=512, block=64, cached=4096, new=1024, ragged=True),
        # The seven drafted rows of one episode at the headline shape (32 heads of 128, no grouping).
        dict(name="rope_7", kind="rope", rows=7, q_heads=32, kv_heads=32, head_dim=128, rotary=128, layout="half",
             scaling="none", span=512, inverse=False, dtype="bf16"),
        # A packed prompt batch of a grouped-head model, positions stretched to 131072 by parts.
        dict(name="rope_16384", kind="rope", rows=16384, q_heads=32, kv_heads=8, head_dim=128, rotary=128, layout="half",
             scaling="parts", span=131072, inverse=False, dtype="bf16"),
        # The gradient of an interleaved rotation of half the head, odd rows, fp32.
        dict(name="rope_back_1023", kind="rope", rows=1023, q_heads=16, kv_heads=4, head_dim=128, rotary=64,
             layout="interleaved", scaling="linear", span=8192, inverse=True, dtype="f32"),
        # Sixteen episodes append seven rows each behind ragged prefixes, fp32 rows as the decoder makes them.
        dict(name="append_16x7", kind="append", batch=16, block=16, cached=532, new=7, ragged=True, kv_heads=32, head_dim=128,
             dtype="f32"),
        # Prompts of up to 4096 tokens into an empty cache.
        dict(name="append_prompts", kind="append", batch=8, block=32, cached=0, new=4096, ragged=True, kv_heads=8,
             head_dim=128, dtype="bf16"),
        # One request, one token, 4000 cached rows: nothing but latency and the split over the context.
        dict(name="decode_1", kind="decode", batch=1, block=16, cached=4000, new=1, ragged=False, q_heads=32, kv_heads=8,
             head_dim=128, dtype="bf16"),
        # Drafts of seven tokens verified for sixteen episodes, one head each, fp16, heads of 64.
        dict(name="decode_16x7", kind="decode", batch=16, block=16, cached=1500, new=7, ragged=True, q_heads=32, kv_heads=32,
             head_dim=64, dtype="f16"),
        # A full batch of long contexts, single tokens: reading the cache.
        dict(name="decode_64_long", kind="decode", batch=64, block=64, cached=8191, new=1, ragged=True, q_heads=32, kv_heads=8,
             head_dim=128, dtype="bf16"),
        # Chunks of at most 276 rows behind ragged pasts, fp16, heads of 64: several requests in one call.
        dict(name="prompt_chunks", kind="prompt", batch=5, past=1500, new=276, ragged=True, q_heads=16, kv_heads=4, head_dim=64,
             causal=True, dtype="f16"),
        # Packed prompts of up to 4096 tokens: the matrix cores' work.
        dict(name="prompt_packed", kind="prompt", batch=8, past=0, new=4096, ragged=True, q_heads=32, kv_heads=8, head_dim=128,
             causal=True, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "rope", "append", "decode", "decode", "decode", "prompt", "prompt", "prompt"])
    if kind == "plan":
        batch = _log(rng, 1, 512)
        return dict(kind=kind, batch=batch, block=rng.choice([16, 32, 64]), cached=_log(rng, 1, 4096), new=_log(rng, 1, 1024),
                    ragged=rng.random() < 0.8)
    head_dim = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16])
    q_heads = kv_heads * rng.choice([g for g in (1, 2, 3, 4, 4, 5, 7, 8) if g * kv_heads <= 32])
    if kind == "rope":
        return dict(kind=kind, rows=_log(rng, 1, 8192), q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim,
                    rotary=rng.choice([head_dim, head_dim, head_dim // 2]), layout=rng.choice(["half", "interleaved"]),
                    scaling=rng.choice(["none", "linear", "base", "parts", "bands"]), span=_log(rng, 64, 131072),
                    inverse=rng.random() < 0.3, dtype=rng.choice(["bf16", "bf16", "f16", "f32"]))
    if kind == "append":
        batch = _log(rng, 1, 64)
        return dict(kind=kind, batch=batch, block=rng.choice([16, 32, 64]), cached=rng.choice([0, _log(rng, 1, 8192 // batch)]),
                    new=_log(rng, 1, 8192 // batch), ragged=rng.random() < 0.7, kv_heads=kv_heads, head_dim=head_dim,
                    dtype=rng.choice(["bf16", "f16", "f32"]))
    if kind == "decode":
        batch = _log(rng, 1, 64)
        new = rng.choice([1, 1, 1, 2, 4, 7, 14])
        cached = _log(rng, 1, min(8191 if new == 1 else 2048, 1500000 // (batch * kv_heads))) - 1
        return dict(kind=kind, batch=batch, block=rng.choice([16, 32, 64]), cached=cached, new=new, ragged=rng.random() < 0.6,
                    q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, dtype=rng.choice(["bf16", "bf16", "f16"]))
    batch = _log(rng, 1, 16)
    new = _log(rng, 1, min(2048, 8192 // batch))
    return dict(kind=kind, batch=batch, past=rng.choice([0, 0, _log(rng, 1, 500)]), new=new, ragged=rng.random() < 0.7,
                q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, causal=rng.random() < 0.8,
                dtype=rng.choice(["bf16", "bf16", "f16"]))


# ---- lengths (the case's own) -----------------------------------------------------------------------------------

def _ragged(rng, most):
    """A length of at most `most`, spread over its logarithm."""
    return 0 if most == 0 else min(most, _log(rng, max(1, most // 8), most))


def _lengths(c):
    """Cached and new rows of every request, as lists; a negative cached length gives a finished request's blocks back."""
    rng, b = random.Random("%s %d %d" % (c["kind"], c["batch"], c["new"])), c["batch"]
    past = c["past"] if c["kind"] == "prompt" else c["cached"]
    if not c["ragged"]:
        return [past] * b, [c["new"]] * b
    cached = [_ragged(rng, past) for _ in range(b)]
    if c["kind"] == "decode":
        return cached, [c["new"]] * b
    new = [_ragged(rng, c["new"]) for _ in range(b)]
    if c["kind"] == "plan":
        for i in range(b):
            what = rng.random()
            if what < 0.05:
                cached[i], new[i] = -1, 0
            elif what < 0.75:
                new[i] = 1
    new[rng.randrange(b)] = c["new"]
    return cached, [0 if p < 0 else n for p, n in zip(cached, new)]


def _sums(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


# ---- inputs -----------------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _rows(g, shape, dtype):
    """Rows of queries, keys or values: every channel has a scale of its own, a few stand out."""
    x = torch.randn(shape, generator=g, device=DEV)
    x *= torch.exp(0.5 * torch.randn(shape[-2:], generator=g, device=DEV))
    return x.to(dtype)


def _cell_bytes(c):
    return c["block"] * (c["head_dim"] + c["head_dim"] // 16)


def _cells(c, pool):
    """The four parts of a pool's cells as views: key codes, value codes, key exponents, value exponents."""
    n, h, bs, hd = pool.shape[0], c["kv_heads"], c["block"], c["head_dim"]
    a, e = bs * hd // 2, bs * hd // 32
    return (pool[..., :a].view(n, h, bs, hd // 2), pool[..., a:2 * a].view(n, h, bs // 4, 16, 4, hd // 32),
            pool[..., 2 * a:2 * a + e].view(n, h, bs, hd // 32), pool[..., 2 * a + e:].view(n, h, bs // 4, hd // 32, 4))


def _quantise(x):
    """fp32 [..., head_dim] -> codes [..., head_dim / 2] and exponents [..., head_dim / 32], as bytes."""
    x = x.view(x.shape[:-1] + (-1, GROUP))
    most = x.abs().amax(-1)
    bits = most.view(torch.int32)
    e = ((bits >> 23) - 2 + ((bits & 0x7FFFFF) > 0x400000)).clamp(min=1)
    y = x.abs() * torch.exp2((127 - e).float())[..., None]
    code = sum((y >= s if i % 2 else y > s).to(torch.uint8) for i, s in enumerate(HALF_STEPS))
    code += torch.signbit(x).to(torch.uint8) * 8
    code = code.view(code.shape[:-2] + (-1, 2))
    return code[..., 0] | code[..., 1] << 4, e.to(torch.uint8)


def _values(code, e):
    """The fp32 values that codes and exponents stand for."""
    level = torch.tensor(LEVELS, device=DEV)
    level = torch.cat([level, -level])
    x = torch.stack([level[(code & 15).long()], level[(code >> 4).long()]], -1).flatten(-2)
    return (x.view(x.shape[:-1] + (-1, GROUP)) * torch.exp2(e.float() - 127)[..., None]).flatten(-2)


def _unpack(c, cells):
    """Whole cells [..., kv_heads, bytes] -> keys and values [..., kv_heads, block, head_dim], fp32."""
    flat = cells.view((-1,) + cells.shape[-2:])
    kc, vc, ke, ve = _cells(c, flat)
    n, h, bs = flat.shape[0], c["kv_heads"], c["block"]
    shape = cells.shape[:-2] + (h, bs, c["head_dim"])
    vc, ve = vc.transpose(3, 4).reshape(n, h, bs, -1), ve.transpose(3, 4).reshape(n, h, bs, -1)
    return _values(kc, ke).view(shape), _values(vc, ve).view(shape)


def _fill(c, g, n_blocks):
    """A pool whose every block holds rows of the usual distribution, a slice of blocks at a time."""
    pool = torch.empty((n_blocks, c["kv_heads"], _cell_bytes(c)), dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 25) // (c["kv_heads"] * c["block"] * c["head_dim"]))
    for i in range(0, n_blocks, step):
        part = pool[i:i + step]
        kc, vc, ke, ve = _cells(c, part)
        shape = (part.shape[0], c["kv_heads"], c["block"], c["head_dim"])
        code, e = _quantise(torch.randn(shape, generator=g, device=DEV))
        kc.copy_(code)
        ke.copy_(e)
        code, e = _quantise(torch.randn(shape, generator=g, device=DEV))
        vc.copy_(code.view(code.shape[:2] + (-1, 4, 16, c["head_dim"] // 32)).transpose(3, 4))
        ve.copy_(e.view(e.shape[:2] + (-1, 4, c["head_dim"] // 32)).transpose(3, 4))
    return pool


def _paged(c, g, total, s):
    """Tables of shuffled blocks for requests of `total` rows."""
    need = [-(-n // c["block"]) for n in total]
    s.n_blocks, s.max_blocks = sum(need) + 3, max(1, max(need))
    order = torch.randperm(s.n_blocks, generator=g, device=DEV).to(torch.int32)
    s.table = torch.full((c["batch"], s.max_blocks), -1, dtype=torch.int32, device=DEV)
    at = _sums(need)
    for i, n in enumerate(need):
        s.table[i, :n] = order[at[i]:at[i] + n]
    s.seq_len, s.cu_seq = _i32(total), _i32(_sums(total))


def _rope_scaling(c):
    """What a model's configuration says about positions."""
    return dict(base=10000.0 if c["scaling"] in ("none", "linear") else 500000.0, factor=1.0 if c["scaling"] == "none" else 8.0,
                original=8192, fast=32.0, slow=1.0, low=1.0, high=4.0)


def prepare(case, seed):
    c, g = case, _gen(seed * 8 + 1)
    s = SimpleNamespace(case=c, call=None)
    if c["kind"] == "rope":
        dt = DTYPES[c["dtype"]]
        s.q = _rows(g, (c["rows"], c["q_heads"], c["head_dim"]), dt)
        s.k = _rows(g, (c["rows"], c["kv_heads"], c["head_dim"]), dt)
        start = torch.randint(0, c["span"], (1,), generator=g, device=DEV)
        s.position = ((start + torch.arange(c["rows"], device=DEV)) % c["span"]).to(torch.int32)
        s.q_out, s.k_out = torch.empty_like(s.q), torch.empty_like(s.k)
        return s
    cached, new = _lengths(c)
    s.rows, s.max_new = sum(new), max(new)
    s.cu_rows = _i32(_sums(new))
    if c["kind"] == "plan":
        b, bs = c["batch"], c["block"]
        held = [-(-(p if p >= 0 else c["cached"] // 2) // bs) for p in cached]
        s.max_blocks = -(-(max(1, c["cached"]) + c["new"]) // bs)
        s.n_blocks = sum(held) + sum(-(-n // bs) + 1 for n in new)
        order = torch.randperm(s.n_blocks, generator=g, device=DEV).to(torch.int32)
        s.table = torch.full((b, s.max_blocks), -1, dtype=torch.int32, device=DEV)
        at = _sums(held)
        for i, n in enumerate(held):
            s.table[i, :n] = order[at[i]:at[i] + n]
        s.free_ids = torch.cat([order[at[-1]:], torch.full((at[-1],), -1, dtype=torch.int32, device=DEV)])
        s.free_count, s.owned = _i32([s.n_blocks - at[-1]]), _i32(held)
        s.cached, s.new = _i32(cached), _i32(new)
        s.rows += 3                                              # a padded batch: three rows belong to nobody
        i32 = dict(dtype=torch.int32, device=DEV)
        s.out = {"table": s.table, "free_ids": s.free_ids, "free_count": torch.empty(1, **i32), "owned": torch.empty(b, **i32),
                 "seq_len": torch.empty(b, **i32), "cu_rows": torch.empty(b + 1, **i32), "cu_seq": torch.empty(b + 1, **i32),
                 "slot": torch.empty(s.rows, **i32), "position": torch.empty(s.rows, **i32)}
        return s
    dt = DTYPES[c["dtype"]]
    total = [p + n for p, n in zip(cached, new)]
    if c["kind"] == "prompt":
        s.q = _rows(g, (s.rows, c["q_heads"], c["head_dim"]), dt)
        s.k, s.v = (_rows(g, (sum(total), c["kv_heads"], c["head_dim"]), dt) for _ in range(2))
        s.cu_seq, s.max_seq = _i32(_sums(total)), max(total)
        s.out = torch.empty_like(s.q)
        s.lse = torch.empty((s.rows, c["q_heads"]), device=DEV)
        return s
    _paged(c, g, total, s)
    s.max_seq, s.total = max(total), sum(total)
    s.pool = _fill(c, g, s.n_blocks)
    if c["kind"] == "append":
        s.k, s.v = (_rows(g, (s.rows, c["kv_heads"], c["head_dim"]), dt) for _ in range(2))
        owner = torch.repeat_interleave(torch.arange(c["batch"], device=DEV), _i32(new).long())
        pos = torch.arange(s.rows, device=DEV) - s.cu_rows[owner] + _i32(cached)[owner]
        s.slot = (s.table[owner, pos // c["block"]] * c["block"] + pos % c["block"]).to(torch.int32)
        s.k_out, s.v_out = (torch.empty((s.total, c["kv_heads"], c["head_dim"]), dtype=dt, device=DEV) for _ in range(2))
        return s
    s.q = _rows(g, (s.rows, c["q_heads"], c["head_dim"]), dt)
    s.out = torch.empty_like(s.q)
    s.lse = torch.empty((s.rows, c["q_heads"]), device=DEV)
    return s


# ---- the library's calls ------------------------------------------------------------------------------------------

def _descriptors(P, s):
    """What a user's program sets up once and hands to every call: descriptors, the rotary table, the workspace."""
    c, h = s.case, SimpleNamespace(P=P)
    if c["kind"] == "plan":
        o = s.out
        h.plan = P.make_plan_desc(block_size=c["block"], n_blocks=s.n_blocks, cached_len=s.cached, new_len=s.new, owned_in=s.owned,
                                  owned_out=o["owned"], block_table=s.table, free_ids=s.free_ids, free_count_in=s.free_count,
                                  free_count_out=o["free_count"], seq_len=o["seq_len"], cu_rows=o["cu_rows"], cu_seq=o["cu_seq"],
                                  slot=o["slot"], position=o["position"])
    elif c["kind"] == "rope":
        r = _rope_scaling(c)
        desc = P.make_rope_desc(rotary_dim=c["rotary"], base=r["base"], scaling=c["scaling"], factor=r["factor"],
                                original_len=r["original"], beta_fast=r["fast"], beta_slow=r["slow"], low_freq=r["low"],
                                high_freq=r["high"])
        h.turns, h.magnitude = P.rope_table(desc, DEV)
        h.q, h.k, h.q_out, h.k_out = (P.head_rows(t) for t in (s.q, s.k, s.q_out, s.k_out))
    elif c["kind"] == "prompt":
        h.q, h.k, h.v, h.out = (P.head_rows(t) for t in (s.q, s.k, s.v, s.out))
    else:
        h.cache = P.make_kv4_desc(s.pool, c["block"], c["kv_heads"], c["head_dim"])
        h.batch = P.make_paged_batch(s.table, s.seq_len, s.cu_rows, s.rows)
        if c["kind"] == "append":
            h.k, h.v, h.k_out, h.v_out = (P.head_rows(t) for t in (s.k, s.v, s.k_out, s.v_out))
        else:
            h.q, h.out = P.head_rows(s.q), P.head_rows(s.out)
            n = P.heisd_kv4_attention_workspace_bytes(h.cache, c["batch"], s.rows, c["q_heads"], s.max_new, s.max_seq)
            h.workspace = torch.empty(n, dtype=torch.uint8, device=DEV)
    return h


def _own(s):
    if s.call is None:
        import paper_2603_17573_amd as P
        s.call = _descriptors(P, s)
    c, h = s.case, s.call
    P, st = h.P, torch.cuda.current_stream().cuda_stream
    if c["kind"] == "plan":
        rc, out = P.heisd_paged_plan(h.plan, st), s.out
    elif c["kind"] == "rope":
        rc = P.heisd_rope(h.turns.data_ptr(), h.magnitude, c["rotary"], P.ROPE_LAYOUT[c["layout"]], c["inverse"],
                          s.position.data_ptr(), c["rows"], c["head_dim"], h.q, h.q_out, h.k, h.k_out, st)
        out = {"q": s.q_out, "k": s.k_out}
    elif c["kind"] == "append":
        rc = P.heisd_kv4_append(h.cache, h.k, h.v, s.slot.data_ptr(), s.rows, st)
        rc = rc or P.heisd_kv4_gather(h.cache, h.batch, s.cu_seq.data_ptr(), s.total, h.k_out, h.v_out, st)
        out = {"k": s.k_out, "v": s.v_out}
    elif c["kind"] == "decode":
        rc = P.heisd_kv4_attention(h.cache, h.batch, h.q, h.out, s.lse.data_ptr(), 1 / math.sqrt(c["head_dim"]), s.max_new,
                                   s.max_seq, h.workspace.data_ptr(), h.workspace.numel(), st)
        out = {"out": s.out, "lse": s.lse}
    else:
        rc = P.heisd_prompt_attention(h.q, h.k, h.v, h.out, s.lse.data_ptr(), s.cu_rows.data_ptr(), s.cu_seq.data_ptr(), c["batch"],
                                      s.rows, s.k.shape[0], c["head_dim"], 1 / math.sqrt(c["head_dim"]), c["causal"], st)
        out = {"out": s.out, "lse": s.lse}
    if rc != 0:
        raise RuntimeError("%s: %d %s" % (c["kind"], rc, P.heisd_last_error(None)))
    return out


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _plan(s):
    c = s.case
    bs, b = c["block"], c["batch"]
    cached, new, owned, table, free_ids = s.cached.long(), s.new.long().clamp(min=0), s.owned.long(), s.table, s.free_ids
    cu = torch.zeros(b + 1, dtype=torch.int64, device=DEV)
    cu[1:] = new.cumsum(0)
    live = (cached >= 0) & (s.new >= 0) & (cached + new <= s.max_blocks * bs) & (cu[1:] <= s.rows)
    # finished requests give their blocks back, in order
    back = torch.where(cached < 0, owned, 0)
    col = torch.arange(s.max_blocks, device=DEV)
    returned = table[col[None, :] < back[:, None]]
    n_free = s.free_count.long() + returned.numel()
    at = s.free_count.long() + torch.arange(returned.numel(), device=DEV)
    free_ids = free_ids.index_put((at,), returned)
    # first come, first served
    need = torch.where(live, ((cached + new + bs - 1) // bs - owned).clamp(min=0), 0)
    before = need.cumsum(0) - need
    live &= (need == 0) | (before + need <= n_free)
    need = torch.where(live, need, 0)
    fresh = (col >= owned[:, None]) & (col < (owned + need)[:, None])
    pick = n_free - 1 - before[:, None] - (col - owned[:, None])
    table = torch.where(fresh, free_ids[pick.clamp(0, s.n_blocks - 1)], table)
    total = torch.where(live, cached + new, -1)
    cu_seq = torch.zeros(b + 1, dtype=torch.int64, device=DEV)
    cu_seq[1:] = total.clamp(min=0).cumsum(0)
    row = torch.arange(s.rows, device=DEV)
    owner = (row[:, None] >= cu[None, 1:]).sum(1)
    mine = owner.clamp(max=b - 1)
    pos = cached[mine] + row - cu[mine]
    ok = (owner < b) & live[mine]
    slot = torch.where(ok, table[mine, (pos // bs).clamp(0, s.max_blocks - 1)] * bs + pos % bs, -1)
    whole = dict(free_count=n_free - need.sum(), owned=torch.where(cached < 0, 0, owned + need), seq_len=total, cu_rows=cu.clamp(max=s.rows),
                 cu_seq=cu_seq, slot=slot, position=torch.where(ok, pos, -1))
    return dict({k: v.to(torch.int32) for k, v in whole.items()}, table=table, free_ids=free_ids)


def _frequencies(c):
    """Radians per position of every pair, in 64 bits, and what cos and sin are multiplied by."""
    r, n = _rope_scaling(c), c["rotary"]
    i = torch.arange(n // 2, dtype=torch.float64, device=DEV)
    base, factor, size = r["base"], r["factor"], 1.0
    if c["scaling"] == "base":
        base = base * factor ** (n / (n - 2))
    freq = base ** (-2 * i / n)
    if c["scaling"] == "linear":
        freq = freq / factor
    elif c["scaling"] == "parts":                                # pairs that turn often keep their speed, slow ones are stretched
        def pair(turns):
            return n * math.log(r["original"] / (turns * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(0, math.floor(pair(r["fast"]))), min(n - 1, math.ceil(pair(r["slow"])))
        keep = 1 - ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        freq = freq * keep + freq / factor * (1 - keep)
        size = 0.1 * math.log(factor) + 1
    elif c["scaling"] == "bands":                                # the same by wavelength
        turns = r["original"] * freq / (2 * math.pi)
        keep = ((turns - r["low"]) / (r["high"] - r["low"])).clamp(0, 1)
        freq = freq * keep + freq / factor * (1 - keep)
    return freq, size


def _rope(s):
    c = s.case
    freq, size = _frequencies(c)
    angle = s.position.double()[:, None, None] * freq
    cos, sin = (angle.cos() * size).float(), (angle.sin() * size).float()
    if c["inverse"]:
        sin = -sin
    n = c["rotary"]

    def turn(x):
        y, rest = x[..., :n].float(), x[..., n:].float()
        if c["layout"] == "half":
            a, b = y[..., :n // 2], y[..., n // 2:]
            y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        else:
            a, b = y[..., 0::2], y[..., 1::2]
            y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        return torch.cat([y, rest], -1).to(x.dtype)

    return {"q": turn(s.q), "k": turn(s.k)}


def _pick(s, x):
    """[batch, kv_heads, blocks, block, head_dim] -> the packed rows [total, kv_heads, head_dim]."""
    b, h = x.shape[:2]
    x = x.reshape(b, h, -1, x.shape[-1]).transpose(1, 2)
    keep = torch.arange(x.shape[1], device=DEV)[None, :] < s.seq_len[:, None]
    return x[keep]


def _append(s):
    c = s.case
    kc, vc, ke, ve = _cells(c, s.pool)
    blk, off = s.slot.long() // c["block"], s.slot.long() % c["block"]
    code, e = _quantise(s.k.float())
    kc[blk, :, off], ke[blk, :, off] = code, e
    code, e = _quantise(s.v.float())
    vc[blk, :, off // 4, :, off % 4] = code.view(code.shape[:2] + (16, -1))
    ve[blk, :, off // 4, :, off % 4] = e
    k, v = _unpack(c, s.pool[s.table.clamp(min=0).long()])       # [batch, blocks, kv_heads, block, head_dim]
    return {"k": _pick(s, k.transpose(1, 2)).to(s.k.dtype), "v": _pick(s, v.transpose(1, 2)).to(s.v.dtype)}


def _attend(q, k, v, seen, scale):
    """q [B, Hk, G * Lq, d], k and v [B, Hk, Lk, d], seen [B, 1, G * Lq, Lk]; out and log of the sum of exponentials."""
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale)
    x.masked_fill_(~seen, -math.inf)
    m = x.amax(-1, keepdim=True).clamp(min=-3e38)
    x = x.sub_(m).exp_()
    n = x.sum(-1, keepdim=True)
    out = torch.matmul(x, v) / n.clamp(min=1e-30)
    return torch.where(n > 0, out, 0), (n.log() + m).squeeze(-1)


def _padded(cu, most):
    """Row numbers [B, most] of packed sequences, and which of them exist."""
    at = torch.arange(most, device=DEV)[None, :]
    there = at < (cu[1:] - cu[:-1])[:, None]
    return torch.where(there, cu[:-1, None] + at, 0).long(), there


def _attention(s, k, v, seq_len, causal):
    """k and v [B, Hk, Lk, d], padded; queries are packed and end where their request's keys end."""
    c = s.case
    hk, grp, hd = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["head_dim"]
    row, there = _padded(s.cu_rows, s.max_new)
    b, lq = row.shape
    q = s.q.float()[row].view(b, lq, hk, grp, hd).permute(0, 2, 3, 1, 4).reshape(b, hk, grp * lq, hd)
    col, last = torch.arange(k.shape[2], device=DEV), seq_len[:, None].expand(b, lq).long()
    if causal:
        last = last - (s.cu_rows[1:] - s.cu_rows[:-1])[:, None] + torch.arange(lq, device=DEV) + 1
    seen = (col[None, None, :] < last[:, :, None]).repeat(1, grp, 1)[:, None]
    out, lse = _attend(q, k, v, seen, 1 / math.sqrt(hd))
    out = out.view(b, hk, grp, lq, hd).permute(0, 3, 1, 2, 4).reshape(b, lq, hk * grp, hd)
    return {"out": out[there].to(s.q.dtype), "lse": lse.view(b, hk, grp, lq).permute(0, 3, 1, 2).reshape(b, lq, -1)[there]}


def _decode(s):
    c = s.case
    k, v = _unpack(c, s.pool[s.table.clamp(min=0).long()])
    k, v = (x.transpose(1, 2).reshape(c["batch"], c["kv_heads"], -1, c["head_dim"]) for x in (k, v))
    return _attention(s, k, v, s.seq_len, True)


def _prompt(s):
    row, _ = _padded(s.cu_seq, s.max_seq)
    k, v = (x.float()[row].transpose(1, 2).contiguous() for x in (s.k, s.v))
    return _attention(s, k, v, s.cu_seq[1:] - s.cu_seq[:-1], s.case["causal"])


def run(state):
    if own:
        return _own(state)
    return {"plan": _plan, "rope": _rope, "append": _append, "decode": _decode, "prompt": _prompt}[state.case["kind"]](state)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------

def work(case):
    c = case
    if c["kind"] == "rope":
        n = c["rows"] * (c["q_heads"] + c["kv_heads"])
        return {"bytes": 2 * n * c["head_dim"] * DTYPES[c["dtype"]].itemsize + c["rows"] * 4 + c["rotary"] * 4, "flops": n * c["rotary"] * 3}
    cached, new = _lengths(c)
    total = [max(0, p) + n for p, n in zip(cached, new)]
    if c["kind"] == "plan":
        blocks = sum(-(-n // c["block"]) for n in total)
        return {"bytes": 4 * (8 * c["batch"] + 2 * blocks + 2 * sum(new)), "flops": 0}
    wide = DTYPES[c["dtype"]].itemsize
    row4 = c["kv_heads"] * (c["head_dim"] + c["head_dim"] // 16)    # a cached row, keys and values
    row = c["kv_heads"] * c["head_dim"] * 2 * wide
    if c["kind"] == "append":
        return {"bytes": sum(new) * (row + row4 + 4) + sum(total) * (row4 + row), "flops": 0}
    pairs = sum(n * t - (n * (n - 1) // 2 if c.get("causal", True) else 0) for n, t in zip(new, total))
    io = sum(new) * c["q_heads"] * (2 * c["head_dim"] * wide + 4)
    return {"bytes": io + sum(total) * (row4 if c["kind"] == "decode" else row), "flops": 4 * pairs * c["q_heads"] * c["head_dim"]}


# ---- the same in 64 bits, written apart --------------------------------------------------------------------------------

def _exact_code(x):
    """The values that rows of 64-bit numbers are held as: the nearest of the sixteen, the even code among equals."""
    flat = x.reshape(-1, GROUP)
    out = torch.empty_like(flat)
    grid = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7], device=DEV)    # even codes first: argmin takes the first of equals
    level = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=DEV)[grid]
    for i in range(0, flat.shape[0], 1 << 17):
        y = flat[i:i + (1 << 17)]
        unit = torch.ldexp(torch.ones_like(y[:, :1]), torch.ceil(torch.log2(y.abs().amax(1, keepdim=True) / 6)).clamp(min=-126))
        out[i:i + (1 << 17)] = level[(y[..., None].abs() / unit[..., None] - level).abs().argmin(-1)] * unit * torch.sign(y)
    return out.view(x.shape)


def _exact_rows(s, i, n):
    """The first n cached rows of request i: keys, values [kv_heads, n, head_dim] in 64 bits."""
    c = s.case
    h, bs, hd = c["kv_heads"], c["block"], c["head_dim"]
    cell = s.pool[s.table[i, :-(-n // bs)].long()].transpose(0, 1)           # [kv_heads, blocks, bytes]
    t, d = torch.arange(bs, device=DEV)[:, None], torch.arange(hd, device=DEV)[None, :]
    per, end, got = hd // 16, bs * hd, []
    at_k = t * (hd // 2) + d // 2
    at_v = bs * hd // 2 + ((t // 4) * 16 + d // per) * (hd // 8) + (t % 4) * (per // 2) + d % per // 2
    e_k = end + t * (hd // 32) + d // 32
    e_v = end + bs * hd // 32 + ((t // 4) * (hd // 32) + d // 32) * 4 + t % 4
    for at, e in ((at_k, e_k), (at_v, e_v)):
        code = cell[..., at].int() >> (4 * (d % 2)) & 15
        m, x = code & 1, code >> 1 & 3
        size = torch.where(x == 0, m * 0.5, (1 + 0.5 * m) * torch.exp2(x.double() - 1))
        size = torch.where(code >= 8, -size, size) * torch.exp2(cell[..., e].double() - 127)
        got.append(size.reshape(h, -1, hd)[:, :n])
    return got


def exact(case, seed):
    c = case
    if c["kind"] == "plan":
        return None                                              # whole numbers
    s = prepare(c, seed)
    if c["kind"] == "rope":
        freq, size = _frequencies(c)
        n = c["rotary"]
        turn = torch.polar(torch.full_like(freq, size)[None].repeat(c["rows"], 1), s.position.double()[:, None] * freq)[:, None]
        turn = turn.conj() if c["inverse"] else turn
        got = {}
        for name, x in (("q", s.q.double()), ("k", s.k.double())):
            y = x[..., :n]
            pairs = torch.complex(y[..., :n // 2], y[..., n // 2:]) if c["layout"] == "half" else torch.view_as_complex(
                y.reshape(y.shape[:-1] + (n // 2, 2)).contiguous())
            pairs = pairs * turn
            y = torch.cat([pairs.real, pairs.imag], -1) if c["layout"] == "half" else torch.view_as_real(pairs).flatten(-2)
            got[name] = torch.cat([y, x[..., n:]], -1)
        return got
    cached, new = _lengths(c)
    total, at, at_seq = [p + n for p, n in zip(cached, new)], _sums(new), _sums([p + n for p, n in zip(cached, new)])
    if c["kind"] == "append":
        parts = {"k": [], "v": []}
        for i in range(c["batch"]):
            old = _exact_rows(s, i, cached[i]) if cached[i] else [torch.empty((c["kv_heads"], 0, c["head_dim"]), device=DEV).double()] * 2
            for name, o, x in (("k", old[0], s.k), ("v", old[1], s.v)):
                parts[name] += [o.transpose(0, 1), _exact_code(x[at[i]:at[i + 1]].double())]
        return {name: torch.cat(p) for name, p in parts.items()}
    out = torch.zeros((s.rows, c["q_heads"], c["head_dim"]), dtype=torch.float64, device=DEV)
    lse = torch.full((s.rows, c["q_heads"]), -math.inf, dtype=torch.float64, device=DEV)
    group = c["q_heads"] // c["kv_heads"]
    for i in range(c["batch"]):
        if c["kind"] == "decode":
            k, v = _exact_rows(s, i, total[i])
        else:
            k, v = (x[at_seq[i]:at_seq[i + 1]].double().transpose(0, 1).contiguous() for x in (s.k, s.v))
        q = s.q[at[i]:at[i + 1]].double().transpose(0, 1).contiguous()
        keep = torch.ones((new[i], total[i]), dtype=torch.bool, device=DEV)
        if c.get("causal", True):
            keep = keep.tril(cached[i])
        for h in range(c["q_heads"]):
            x = (q[h] @ k[h // group].T.contiguous()) / math.sqrt(c["head_dim"])
            x = x.masked_fill(~keep, -math.inf)
            lse[at[i]:at[i + 1], h] = torch.logsumexp(x, -1)
            out[at[i]:at[i + 1], h] = torch.softmax(x, -1) @ v[h // group]
    return {"out": out, "lse": lse}
