"""Continuations that share a context, and a cache that is kept small: five operators as measurable cases, with their plain forms.

select   beam search's choice of the next beams over beams and vocabulary (heisd_beam_select)
fork     requests continue others: block tables by parents, and the cached rows that have to be copied (heisd_paged_reorder,
         heisd_kv4_copy), read back (heisd_kv4_gather)
shared   attention of groups of requests over a prefix that a group shares, and over the requests' own tokens (heisd_kv4_shared_attention)
weigh    the attention weight of every cached token, added up over rows and steps (heisd_kv4_weigh)
evict    the heaviest and the latest tokens stay in the cache, in every layer and head (heisd_kv4_evict), read back (heisd_kv4_gather)

Where `own` is false run() is elementary torch in 32 bits (scores of beams in 64, whole numbers in 64); where it is true it
makes the library's calls.  Lengths belong to a case, values (parents and weights among them) to a seed.

The cache: a pool of blocks of block_size tokens.  Every group of 32 values of a row is held as 4-bit floats (sign, two bits
of exponent, one of mantissa: 0 .5 1 1.5 2 3 4 6) times a power of two, the smallest for which the largest value is at most
6, kept as its exponent plus 127 in a byte.  One block of one head is a cell of bytes: key codes [token][head_dim / 2], value
codes [token / 4][16][token % 4][head_dim / 32], key exponents [token][head_dim / 32], value exponents
[token / 4][head_dim / 32][token % 4]; in a byte of codes the low half comes first.  Weights are fp32 [n_blocks][kv_heads][block_size].
"""
import math
import random
from types import SimpleNamespace

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
GROUP = 32
HALF_STEPS = (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)             # between neighbouring 4-bit values
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # One episode, four beams over the 256 action bins, fp32 logits as the decoder gives them: launch latency.
        dict(name="select_1x4", kind="select", groups=1, beams=4, width=4, vocab=256, dtype="f32", power=0.0, finished=False),
        # Sixteen requests of four beams over a vocabulary of 32000, some beams finished, scores by length.
        dict(name="select_16x4", kind="select", groups=16, beams=4, width=4, vocab=32000, dtype="bf16", power=0.6, finished=True),
        # Sixty-four requests of eight beams over a large vocabulary of odd size: reading the logits.
        dict(name="select_64x8", kind="select", groups=64, beams=8, width=8, vocab=131071, dtype="f16", power=0.0, finished=True),
        # Four beams behind one prefix, eight tokens each, two layers: launches.
        dict(name="fork_1x4", kind="fork", groups=1, beams=4, block=16, cached=8, layers=2, kv_heads=32, head_dim=128),
        # Sixteen requests of eight beams with up to 500 tokens of their own.
        dict(name="fork_16x8", kind="fork", groups=16, beams=8, block=64, cached=500, layers=2, kv_heads=8, head_dim=128),
        # Four candidates of one episode behind its 276-row prefix, no grouping of heads: latency.
        dict(name="shared_1x4", kind="shared", groups=1, members=4, prefix=276, cached=7, new=1, block=16, q_heads=32, kv_heads=32,
             head_dim=128, dtype="bf16"),
        # Eight prompts with eight beams each, fp16, heads of 64.
        dict(name="shared_8x8", kind="shared", groups=8, members=8, prefix=4000, cached=63, new=1, block=64, q_heads=32, kv_heads=8,
             head_dim=64, dtype="f16"),
        # Two long contexts with sixty-four continuations each that verify drafts of seven tokens: the matrix cores' work.
        dict(name="shared_2x64x7", kind="shared", groups=2, members=64, prefix=8191, cached=121, new=7, block=64, q_heads=32,
             kv_heads=8, head_dim=128, dtype="bf16"),
        # Weights of four shared contexts from sixteen single tokens each.
        dict(name="weigh_4x16", kind="weigh", groups=4, members=16, prefix=4095, cached=60, new=1, block=64, q_heads=16, kv_heads=4,
             head_dim=64, dtype="f16"),
        # A full batch of long contexts of their own, single tokens: reading the keys.
        dict(name="weigh_64", kind="weigh", groups=64, members=1, prefix=0, cached=8191, new=1, block=64, q_heads=32, kv_heads=8,
             head_dim=128, dtype="bf16"),
        # One context at its budget: 64 of 2112 tokens go, the last 64 stay, two layers.
        dict(name="evict_1", kind="evict", batch=1, block=16, cached=2112, ragged=False, keep=2048, recent=64, layers=2, kv_heads=8,
             head_dim=128),
        # Sixteen prompts of up to 8192 tokens are cut to 1024.
        dict(name="evict_16", kind="evict", batch=16, block=64, cached=8192, ragged=True, keep=1024, recent=128, layers=1, kv_heads=8,
             head_dim=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["select", "select", "fork", "shared", "shared", "shared", "weigh", "weigh", "evict"])
    if kind == "select":
        groups, beams = _log(rng, 1, 64), rng.choice([1, 2, 3, 4, 5, 8, 16])
        return dict(kind=kind, groups=groups, beams=beams, width=rng.choice([beams, beams, rng.randint(1, 16)]),
                    vocab=_log(rng, 100, min(131071, 30000000 // (groups * beams))), dtype=rng.choice(["bf16", "f16", "f32"]),
                    power=rng.choice([0.0, 0.6, 1.0]), finished=rng.random() < 0.5)
    head_dim = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16])
    if kind == "fork":
        groups, beams = _log(rng, 1, 16), rng.choice([2, 3, 4, 8])
        return dict(kind=kind, groups=groups, beams=beams, block=rng.choice([16, 32, 64]), cached=_log(rng, 1, 4000 // (groups * beams) + 8),
                    layers=rng.choice([1, 2, 3]), kv_heads=kv_heads, head_dim=head_dim)
    if kind == "evict":
        batch = _log(rng, 1, 32)
        cached = _log(rng, 32, min(8192, 65536 // batch))
        keep = _log(rng, 1, cached)
        return dict(kind=kind, batch=batch, block=rng.choice([16, 32, 64]), cached=cached, ragged=rng.random() < 0.6, keep=keep,
                    recent=rng.choice([0, _log(rng, 1, keep)]), layers=rng.choice([1, 1, 2]), kv_heads=kv_heads, head_dim=head_dim)
    q_heads = kv_heads * rng.choice([g for g in (1, 2, 3, 4, 4, 5, 7, 8) if g * kv_heads <= 32])
    groups, members, new = _log(rng, 1, 8), _log(rng, 1, 64), rng.choice([1, 1, 1, 2, 4, 7])
    if kind == "weigh" and rng.random() < 0.4:
        batch = _log(rng, 1, 64)
        return dict(kind=kind, groups=batch, members=1, prefix=0, cached=_log(rng, 1, min(8191, 100000 // batch)), new=new,
                    block=rng.choice([16, 32, 64]), q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim,
                    dtype=rng.choice(["bf16", "bf16", "f16"]))
    return dict(kind=kind, groups=groups, members=members, prefix=_log(rng, 1, min(8191, 24000 // groups)),
                cached=_log(rng, 1, min(1024, 16000 // (groups * members))) - 1, new=new, block=rng.choice([16, 32, 64]), q_heads=q_heads,
                kv_heads=kv_heads, head_dim=head_dim, dtype=rng.choice(["bf16", "bf16", "f16"]))


# ---- lengths (the case's own) -----------------------------------------------------------------------------------

def _ragged(rng, most):
    """A length of at most `most`, spread over its logarithm."""
    return 0 if most == 0 else min(most, _log(rng, max(1, most // 8), most))


def _sums(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def _lengths(c):
    """Tokens of every row of the block table, as a list.  fork: a group's beams have the same; shared and weigh: the members' own,
    the rows of this step included, then the prefixes'."""
    rng = random.Random("%s %d %d" % (c["kind"], c["block"], c["cached"]))
    if c["kind"] == "fork":
        return [n for n in (_ragged(rng, c["cached"]) for _ in range(c["groups"])) for _ in range(c["beams"])]
    if c["kind"] == "evict":
        return [_ragged(rng, c["cached"]) if c["ragged"] else c["cached"] for _ in range(c["batch"] - 1)] + [c["cached"]]
    own_tokens = [_ragged(rng, c["cached"]) + c["new"] for _ in range(c["groups"] * c["members"])]
    return own_tokens + [_ragged(rng, c["prefix"]) for _ in range(c["groups"] if c["prefix"] else 0)]


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
    """Tables of shuffled blocks for requests of `total` tokens; the blocks that are left are free."""
    need = [-(-n // c["block"]) for n in total]
    s.n_blocks, s.max_blocks = sum(need) + 3, max(1, max(need))
    order = torch.randperm(s.n_blocks, generator=g, device=DEV).to(torch.int32)
    at, n = _i32(_sums(need)[:-1])[:, None], _i32(need)[:, None]
    col = torch.arange(s.max_blocks, device=DEV)[None, :]
    s.table = torch.where(col < n, order[(at + col).clamp(max=s.n_blocks - 1).long()], -1)
    s.seq_len, s.owned = _i32(total), _i32(need)
    s.free_ids = torch.cat([order[sum(need):], torch.full((sum(need),), -1, dtype=torch.int32, device=DEV)])
    s.free_count = _i32([3])


def _select_state(c, g, s):
    rows = c["groups"] * c["beams"]
    s.logits = (2.5 * torch.randn((rows, c["vocab"]), generator=g, device=DEV)).to(DTYPES[c["dtype"]])
    s.score = -12 * torch.rand(rows, generator=g, device=DEV)
    steps = torch.randint(1, 40, (c["groups"], 1), generator=g, device=DEV).expand(-1, c["beams"]).reshape(-1)
    done = torch.rand(rows, generator=g, device=DEV) < (0.2 if c["finished"] else 0)
    s.length = torch.where(done, (steps * torch.rand(rows, generator=g, device=DEV)).long() + 1, steps + 1).to(torch.int32)
    s.done, s.end = done.to(torch.int32), 2 if c["finished"] else -1
    shape = (c["groups"], c["width"])
    s.out = {k: torch.empty(shape, dtype=torch.int32, device=DEV) for k in ("beam", "token", "length", "done")}
    s.out["score"] = torch.empty(shape, device=DEV)


def prepare(case, seed):
    c, g = case, _gen(seed * 8 + 3)
    s = SimpleNamespace(case=c, call=None)
    if c["kind"] == "select":
        _select_state(c, g, s)
        return s
    total = _lengths(c)
    _paged(c, g, total, s)
    layers, b = c.get("layers", 1), len(total)
    i32 = dict(dtype=torch.int32, device=DEV)
    s.pool = torch.stack([_fill(c, g, s.n_blocks) for _ in range(layers)])
    if c["kind"] == "fork":
        beam = torch.randint(0, c["beams"], (c["groups"], c["beams"]), generator=g, device=DEV)
        s.parent = (beam + torch.arange(c["groups"], device=DEV)[:, None] * c["beams"]).reshape(-1).to(torch.int32)
        s.out = {"table": torch.empty((b, s.max_blocks), **i32), "owned": torch.empty(b, **i32), "length": torch.empty(b, **i32),
                 "copy_from": torch.empty(b, **i32), "free_ids": s.free_ids, "free_count": torch.empty(1, **i32)}
        after = total
    elif c["kind"] == "evict":
        shape = (layers, s.n_blocks, c["kv_heads"], c["block"])
        s.weight = torch.exp(2 * torch.randn(shape, generator=g, device=DEV))
        s.keep = torch.full((b,), c["keep"], **i32)
        s.out = {"weight": torch.zeros_like(s.weight), "length": torch.empty(b, **i32)}
        after = [min(n, c["keep"]) for n in total]
    else:
        dt, m = DTYPES[c["dtype"]], c["groups"] * c["members"]
        s.rows, s.max_own, s.max_prefix = m * c["new"], max(total[:m]), max(total[m:] or [0])
        s.cu_rows = _i32([c["new"] * min(i, m) for i in range(b + 1)])
        s.first = _i32([c["members"] * i for i in range(c["groups"] + 1)])
        s.prefix = _i32([m + i for i in range(c["groups"])])
        s.q = _rows(g, (s.rows, c["q_heads"], c["head_dim"]), dt)
        s.out = {"out": torch.empty_like(s.q), "lse": torch.empty((s.rows, c["q_heads"]), device=DEV)}
        if c["kind"] == "weigh":
            s.lse = _shared(s)["lse"]                            # what the attention of the same rows gave
            s.weight = torch.exp(torch.randn((s.n_blocks, c["kv_heads"], c["block"]), generator=g, device=DEV))
            s.out = {"weight": torch.zeros_like(s.weight)}
        return s
    s.cu_seq, s.total = _i32(_sums(after)), sum(after)
    shape = (layers, 2, s.total, c["kv_heads"], c["head_dim"])
    s.rows_back = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
    return s


# ---- the library's calls ------------------------------------------------------------------------------------------

def _descriptors(P, s):
    """What a user's program sets up once and hands to every call: descriptors and workspaces."""
    c, h, o = s.case, SimpleNamespace(P=P), s.out
    if c["kind"] == "select":
        h.beams = P.make_beam_desc(s.logits, c["beams"], c["width"], s.score, o["score"], o["beam"], o["token"], length_in=s.length,
                                   length_out=o["length"], done_in=s.done, done_out=o["done"], end_token=s.end, length_power=c["power"])
        n = P.heisd_beam_select_workspace_bytes(c["groups"], c["beams"], c["width"], c["vocab"])
        h.workspace = torch.empty(n, dtype=torch.uint8, device=DEV)
        return h
    h.caches = [P.make_kv4_desc(p, c["block"], c["kv_heads"], c["head_dim"]) for p in s.pool]
    h.layers, h.layer_bytes = len(s.pool), s.pool[0].numel()
    if c["kind"] in ("fork", "evict"):
        h.back = [(P.head_rows(r[0]), P.head_rows(r[1])) for r in s.rows_back]
        if c["kind"] == "fork":
            h.books = P.make_reorder_desc(c["block"], s.n_blocks, s.parent, s.seq_len, s.owned, s.table, o["length"], o["owned"], o["table"],
                                          o["copy_from"], s.free_ids, s.free_count, o["free_count"])
        else:
            h.before = P.make_paged_batch(s.table, s.seq_len, None, 0)
        h.batch = P.make_paged_batch(o.get("table", s.table), o["length"], None, 0)
        return h
    h.batch = P.make_paged_batch(s.table, s.seq_len, s.cu_rows, s.rows)
    h.groups = P.make_prefix_groups(s.first, s.prefix, c["members"] * c["new"], s.max_prefix) if c["prefix"] else None
    h.q = P.head_rows(s.q)
    if c["kind"] == "shared":
        h.out = P.head_rows(o["out"])
        n = P.heisd_kv4_shared_attention_workspace_bytes(h.caches[0], len(s.seq_len), s.rows, c["q_heads"], c["new"], s.max_own, h.groups)
        h.workspace = torch.empty(n, dtype=torch.uint8, device=DEV)
    return h


def _own(s):
    if s.call is None:
        import paper_2603_17573_amd as P
        s.call = _descriptors(P, s)
    c, h, o = s.case, s.call, s.out
    P, st = h.P, torch.cuda.current_stream().cuda_stream
    if c["kind"] == "select":
        rc = P.heisd_beam_select(h.beams, h.workspace.data_ptr(), h.workspace.numel(), st)
    elif c["kind"] == "shared":
        rc = P.heisd_kv4_shared_attention(h.caches[0], h.batch, h.groups, h.q, h.out, o["lse"].data_ptr(), 1 / math.sqrt(c["head_dim"]),
                                          c["new"], s.max_own, h.workspace.data_ptr(), h.workspace.numel(), st)
    elif c["kind"] == "weigh":
        rc = P.heisd_kv4_weigh(h.caches[0], h.batch, h.groups, h.q, s.lse.data_ptr(), 1 / math.sqrt(c["head_dim"]), DECAY,
                               s.weight.data_ptr(), o["weight"].data_ptr(), s.max_own, st)
    else:
        if c["kind"] == "fork":
            rc = P.heisd_paged_reorder(h.books, st)
            rc = rc or P.heisd_kv4_copy(h.caches[0], h.layers, h.layer_bytes, h.batch, o["copy_from"].data_ptr(), None, c["cached"], st)
        else:
            rc = P.heisd_kv4_evict(h.caches[0], h.layers, h.layer_bytes, h.before, s.keep.data_ptr(), c["recent"], s.weight.data_ptr(),
                                   o["weight"].data_ptr(), o["length"].data_ptr(), c["cached"], st)
        for cache, (k, v) in zip(h.caches, h.back):
            rc = rc or P.heisd_kv4_gather(cache, h.batch, s.cu_seq.data_ptr(), s.total, k, v, st)
        o = dict(o, rows=s.rows_back)
    if rc != 0:
        raise RuntimeError("%s: %d %s" % (c["kind"], rc, P.heisd_last_error(None)))
    return o


# ---- plain forms ----------------------------------------------------------------------------------------------------

DECAY = 0.96875                                                  # of a token's weight from one step to the next


def _select(s):
    c = s.case
    g, b, v = c["groups"], c["beams"], c["vocab"]
    x = s.logits.double().view(g, b, v)
    m = x.amax(-1, keepdim=True)
    x -= (x - m).exp().sum(-1, keepdim=True).log() + m
    before, length, done = s.score.double().view(g, b), s.length.long().view(g, b), s.done.view(g, b) != 0
    x += before[..., None]
    if s.end >= 0:                                               # a finished beam goes on as it is, in its end token's place
        x.masked_fill_(done[..., None], -math.inf)
        x[..., s.end] = torch.where(done, before, x[..., s.end])
    after = length + (~done).long()
    rank = x / after.double()[..., None] ** c["power"]
    at = rank.view(g, -1).sort(descending=True, stable=True).indices[:, :c["width"]]
    beam, token = at // v, at % v
    score = x.view(g, -1).gather(1, at)
    none = score == -math.inf                                    # fewer candidates than wanted
    out = {"beam": beam.masked_fill(none, -1), "token": token.masked_fill(none, -1), "length": after.gather(1, beam).masked_fill(none, 0),
           "done": done.gather(1, beam) | (token == s.end) | none}
    return dict({k: t.to(torch.int32) for k, t in out.items()}, score=score.float())


def _read_back(s, table, length):
    """Cached rows of every request and layer, packed, bf16: [layers, 2, total, kv_heads, head_dim]."""
    c = s.case
    keep = torch.arange(table.shape[1] * c["block"], device=DEV)[None, :] < length[:, None]
    x = torch.stack(_unpack(c, s.pool[:, table.clamp(min=0).long()]), 1)      # [layers, 2, batch, blocks, kv_heads, block, head_dim]
    x = x.transpose(4, 5).reshape(x.shape[:3] + (-1, c["kv_heads"], c["head_dim"]))
    return x[:, :, keep].to(torch.bfloat16)


def _fork(s):
    c, b, bs = s.case, len(s.parent), s.case["block"]
    parent, owned, length = s.parent.long(), s.owned.long(), s.seq_len.long()
    at, col = torch.arange(b, device=DEV), torch.arange(s.max_blocks, device=DEV)
    key = torch.where(parent == at, -1, at)                      # a parent's own continuation comes first, then the lowest
    first = torch.full((b,), b, device=DEV).scatter_reduce(0, parent, key, "amin")
    heir = first[parent] == key
    # blocks of those that nobody continues go on top of the free ones
    back = torch.where(first == b, owned, 0)
    returned = s.table[col[None, :] < back[:, None]]
    n_free = s.free_count.long() + returned.numel()
    free_ids = s.free_ids.index_put((s.free_count.long() + torch.arange(returned.numel(), device=DEV),), returned)
    # and the other continuations take theirs from there
    need = torch.where(heir, 0, (length[parent] + bs - 1) // bs)
    before = need.cumsum(0) - need
    given = before + need <= n_free
    need = torch.where(given, need, 0)
    pick = (n_free - 1 - before[:, None] - col).clamp(0, s.n_blocks - 1)
    mine = torch.where(heir, owned[parent], need)
    table = torch.where(col < mine[:, None], torch.where(heir[:, None], s.table[parent], free_ids[pick]), -1)
    source = torch.where(first[parent] < 0, parent, first[parent])
    copied = given & ~heir & (length[parent] > 0)
    out = {"table": table, "owned": mine, "length": torch.where(given, length[parent], -1), "copy_from": torch.where(copied, source, -1),
           "free_ids": free_ids, "free_count": n_free - need.sum()}
    out = {k: t.to(torch.int32) for k, t in out.items()}
    there = (col < need[:, None]) & copied[:, None]
    s.pool[:, table[there].long()] = s.pool[:, table[source][there].long()]
    return dict(out, rows=_read_back(s, out["table"], out["length"]))


def _own_rows(s, table, blocks):
    """Keys and values [requests, kv_heads, tokens, head_dim] of some rows of the table."""
    c = s.case
    k, v = _unpack(c, s.pool[0, table[:, :blocks].clamp(min=0).long()])
    return [x.transpose(1, 2).reshape(len(table), c["kv_heads"], -1, c["head_dim"]) for x in (k, v)]


def _scores(s, q, k, seen):
    """q [B, kv_heads, columns, head_dim], k [B, kv_heads, tokens, head_dim], seen [B, 1, columns or 1, tokens]."""
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(1 / math.sqrt(s.case["head_dim"]))
    return x.masked_fill_(~seen, -math.inf)


def _parts(s):
    """Scores and values of the two parts: [groups * members, kv_heads, new * group, own tokens], [groups, kv_heads, members * new * group, prefix]."""
    c = s.case
    g, m, n, hk, hd = c["groups"], c["members"], c["new"], c["kv_heads"], c["head_dim"]
    grp = c["q_heads"] // hk
    q = s.q.float().view(g, m, n, hk, grp, hd)
    k, v = _own_rows(s, s.table[:g * m], -(-s.max_own // c["block"]))
    last = s.seq_len[:g * m, None] - n + torch.arange(n, device=DEV) + 1              # tokens that a row sees
    seen = torch.arange(k.shape[2], device=DEV) < last.repeat_interleave(grp, 1)[:, None, :, None]
    parts = [(_scores(s, q.permute(0, 1, 3, 2, 4, 5).reshape(g * m, hk, n * grp, hd), k, seen), v)]
    if c["prefix"]:
        k, v = _own_rows(s, s.table[g * m:], -(-s.max_prefix // c["block"]))
        seen = (torch.arange(k.shape[2], device=DEV) < s.seq_len[g * m:, None])[:, None, None]
        parts.append((_scores(s, q.permute(0, 3, 1, 2, 4, 5).reshape(g, hk, m * n * grp, hd), k, seen), v))
    return parts


def _by_row(s, x, part):
    """A part's columns as [groups, members, new, kv_heads, group, ...]."""
    c = s.case
    g, m, n, hk = c["groups"], c["members"], c["new"], c["kv_heads"]
    if part == 0:
        return x.reshape((g, m, hk, n, c["q_heads"] // hk) + x.shape[3:]).transpose(2, 3)
    return x.reshape((g, hk, m, n, c["q_heads"] // hk) + x.shape[3:]).permute((0, 2, 3, 1, 4) + tuple(range(5, x.dim() + 2)))


def _by_part(s, x, part):
    """[groups, members, new, kv_heads, group] as a part's columns, with one value each."""
    g, m, n, hk, grp = x.shape
    if part == 0:
        return x.transpose(2, 3).reshape(g * m, hk, n * grp, 1)
    return x.permute(0, 3, 1, 2, 4).reshape(g, hk, m * n * grp, 1)


def _shared(s):
    c, parts = s.case, _parts(s)
    top = torch.stack([_by_row(s, x.amax(-1), i) for i, (x, _) in enumerate(parts)]).amax(0)
    total, out = 0, 0
    for i, (x, v) in enumerate(parts):
        x = x.sub_(_by_part(s, top, i)).exp_()
        total = total + _by_row(s, x.sum(-1), i)
        out = out + _by_row(s, torch.matmul(x, v), i)
    out = out / total[..., None]
    return {"out": out.reshape(s.q.shape).to(s.q.dtype), "lse": (total.log() + top).reshape(s.rows, c["q_heads"])}


def _weigh(s):
    c = s.case
    m, bs, weight = c["groups"] * c["members"], c["block"], s.out["weight"]
    lse = s.lse.view(c["groups"], c["members"], c["new"], c["kv_heads"], -1)
    for i, (x, _) in enumerate(_parts(s)):
        fresh = x.sub_(_by_part(s, lse, i)).exp_().sum(2)                             # [requests, kv_heads, tokens]
        table, length = (s.table[:m], s.seq_len[:m]) if i == 0 else (s.table[m:], s.seq_len[m:])
        t = torch.arange(fresh.shape[2], device=DEV)
        block, there = table[:, t // bs].clamp(min=0).long(), t < length[:, None]
        old = s.weight[block, :, t % bs]                                              # [requests, tokens, kv_heads]
        if i == 0:
            old = torch.where((t < length[:, None] - c["new"])[..., None], old, 0)    # this step's tokens had none
        now = DECAY * old + fresh.transpose(1, 2)
        weight[block[there], :, (t % bs).expand_as(block)[there]] = now[there]
    return {"weight": weight}


def _tokens(c, pool):
    """The bytes of a pool [..., kv_heads, bytes] by token: key codes, value codes, key exponents, value exponents [..., kv_heads, block, bytes]."""
    kc, vc, ke, ve = _cells(c, pool.view((-1,) + pool.shape[-2:]))
    shape = pool.shape[:-1] + (c["block"], -1)
    return [x.reshape(shape) for x in (kc, vc.transpose(3, 4), ke, ve.transpose(3, 4))]


def _evict(s):
    c = s.case
    layers, hk, bs, most = len(s.pool), c["kv_heads"], c["block"], c["keep"]
    table, n = s.table.clamp(min=0).long(), s.seq_len.long()[:, None]
    t = torch.arange(s.max_blocks * bs, device=DEV)
    recent = min(c["recent"], most)
    cut, stay, first = n > most, n - recent, most - recent       # requests that lose tokens; candidates, and how many of them stay
    weight = s.weight[:, table].transpose(2, 3).reshape(layers, len(table), hk, -1)
    rank = torch.where((t < stay)[:, None], weight, -math.inf).sort(dim=-1, descending=True, stable=True).indices.argsort(-1)
    chosen = rank < first
    hole, source = ~chosen & (t < first), chosen & (t >= first)
    # the i-th hole takes the i-th token that stays and lies behind
    filler = (~source).to(torch.uint8).sort(dim=-1, stable=True).indices.gather(-1, (hole.cumsum(-1) - 1).clamp(min=0))
    moved = torch.where(hole, filler, torch.where((t < first), t, (t + n - most).clamp(max=len(t) - 1))[:, None])
    src = torch.where(cut[:, None], moved, t)
    length = n.clamp(max=most)
    there = (t < length)[:, None].expand(-1, hk, -1)              # [batch, kv_heads, tokens]
    block, off = (x[:, None].expand(-1, hk, -1)[there] for x in (table[:, t // bs], (t % bs).expand(len(table), -1)))
    head = torch.arange(hk, device=DEV)[None, :, None].expand_as(there)[there]
    out = s.out["weight"]
    out[:, block, head, off] = weight.gather(-1, src)[:, there]
    cells = s.pool[:, table]
    kc, vc, ke, ve = (x.transpose(2, 3).reshape(layers, len(table), hk, len(t), -1) for x in _tokens(c, cells))
    kc, vc, ke, ve = (x.gather(3, src[..., None].expand_as(x))[:, there] for x in (kc, vc, ke, ve))
    flat = s.pool.view((-1,) + s.pool.shape[-2:])
    a, b, d, e = (x.view((layers, -1) + x.shape[1:]) for x in _cells(c, flat))
    a[:, block, head, off], d[:, block, head, off] = kc, ke
    b[:, block, head, off // 4, :, off % 4] = vc.view(vc.shape[:2] + (16, -1)).movedim(1, 0)
    e[:, block, head, off // 4, :, off % 4] = ve.movedim(1, 0)
    length = length[:, 0].to(torch.int32)
    return {"weight": out, "length": length, "rows": _read_back(s, s.table, length)}


def run(state):
    if own:
        return _own(state)
    return {"select": _select, "fork": _fork, "shared": _shared, "weigh": _weigh, "evict": _evict}[state.case["kind"]](state)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------

def work(case):
    c = case
    if c["kind"] == "select":
        rows = c["groups"] * c["beams"]
        return {"bytes": rows * (c["vocab"] * DTYPES[c["dtype"]].itemsize + 12) + c["groups"] * c["width"] * 20, "flops": rows * c["vocab"] * 4}
    total, layers = _lengths(c), c.get("layers", 1)
    row4 = c["kv_heads"] * (c["head_dim"] + c["head_dim"] // 16)    # a cached row, keys and values
    back = row4 + c["kv_heads"] * c["head_dim"] * 4                 # reading it back into bf16
    blocks = sum(-(-n // c["block"]) for n in total)
    if c["kind"] == "fork":
        gone = (1 - 1 / c["beams"]) ** c["beams"]                   # beams that nobody continues, on average: as many are copied
        return {"bytes": 4 * (8 * len(total) + 3 * blocks) + layers * sum(total) * (2 * gone * row4 + back), "flops": 0}
    if c["kind"] == "evict":
        recent, size = min(c["recent"], c["keep"]), 0.0
        for n in total:
            size += back * min(n, c["keep"])
            if n > c["keep"]:                                       # all weights, what fills the holes, the latest
                first = c["keep"] - recent
                size += 4 * c["kv_heads"] * (n - recent) + 2 * (row4 + 4 * c["kv_heads"]) * (first * (1 - first / max(1, n - recent)) + recent)
        return {"bytes": layers * size + 4 * blocks, "flops": 0}
    m, n = c["groups"] * c["members"], c["new"]
    rows, own_pairs = m * n, sum(n * t - n * (n - 1) // 2 for t in total[:m])
    pairs = own_pairs + sum(c["members"] * n * t for t in total[m:])
    wide = DTYPES[c["dtype"]].itemsize
    if c["kind"] == "shared":
        return {"bytes": rows * c["q_heads"] * (2 * c["head_dim"] * wide + 4) + sum(total) * row4 + 4 * blocks,
                "flops": 4 * pairs * c["q_heads"] * c["head_dim"]}
    return {"bytes": rows * c["q_heads"] * (c["head_dim"] * wide + 4) + sum(total) * (row4 // 2 + 8 * c["kv_heads"]) + 4 * blocks,
            "flops": 2 * pairs * c["q_heads"] * c["head_dim"]}


# ---- the same in 64 bits, written apart --------------------------------------------------------------------------------

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


def _exact_cached(s, layer, i, n):
    return _exact_rows(SimpleNamespace(case=s.case, pool=s.pool[layer], table=s.table), i, n)


def _exact_select(s):
    c, got = s.case, []
    x, before = s.logits.double().cpu().numpy(), s.score.double().cpu().numpy()
    done, length = s.done.cpu().numpy(), s.length.cpu().numpy()
    for g in range(c["groups"]):
        best = []
        for i in range(g * c["beams"], (g + 1) * c["beams"]):
            if done[i]:
                best.append((before[i] / float(length[i]) ** c["power"], before[i]))
                continue
            top = np.partition(x[i], -min(c["width"], c["vocab"]))[-c["width"]:]
            scores = before[i] + top - np.logaddexp.reduce(x[i])
            best += [(v / float(length[i] + 1) ** c["power"], v) for v in scores]
        got.append(([v for _, v in sorted(best, reverse=True)] + [-math.inf] * c["width"])[:c["width"]])
    return torch.tensor(np.array(got), device=DEV)


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["kind"] == "select":
        return {"beam": None, "token": None, "length": None, "done": None, "score": _exact_select(s)}
    total = _lengths(c)
    if c["kind"] in ("fork", "evict"):
        rows = []
        for layer in range(len(s.pool)):
            k, v = [], []
            for i, n in enumerate(total):
                if c["kind"] == "fork":
                    a, b = _exact_cached(s, layer, int(s.parent[i]), n)
                else:
                    a, b = _exact_cached(s, layer, i, n)
                    a, b = _exact_cut(s, layer, i, n, a, b)
                k.append(a.transpose(0, 1))
                v.append(b.transpose(0, 1))
            rows.append(torch.stack([torch.cat(k), torch.cat(v)]))
        none = ("table", "owned", "length", "copy_from", "free_ids", "free_count") if c["kind"] == "fork" else ("weight", "length")
        return dict({k: None for k in none}, rows=torch.stack(rows))
    m, grp, scale = c["groups"] * c["members"], c["q_heads"] // c["kv_heads"], 1 / math.sqrt(c["head_dim"])
    out = torch.empty((s.rows, c["q_heads"], c["head_dim"]), dtype=torch.float64, device=DEV)
    lse = torch.empty((s.rows, c["q_heads"]), dtype=torch.float64, device=DEV)
    weight = torch.zeros((s.n_blocks, c["kv_heads"], c["block"]), dtype=torch.float64, device=DEV)

    def note(i, n, fresh, has):
        t = torch.arange(n, device=DEV)
        at = s.table[i, t // c["block"]].long()
        old = s.weight[at, :, t % c["block"]].double().T * (t < has)
        weight[at, :, t % c["block"]] = (DECAY * old + fresh).T

    for g in range(c["groups"]):
        if c["prefix"]:
            pk, pv = _exact_cached(s, 0, m + g, total[m + g])
        else:
            pk = pv = torch.empty((c["kv_heads"], 0, c["head_dim"]), dtype=torch.float64, device=DEV)
        on_prefix = 0
        for i in range(g * c["members"], (g + 1) * c["members"]):
            ok, ov = _exact_cached(s, 0, i, total[i])
            r = slice(i * c["new"], (i + 1) * c["new"])
            q = s.q[r].double().view(c["new"], c["kv_heads"], grp, -1).permute(1, 2, 0, 3).reshape(c["kv_heads"], -1, c["head_dim"])
            hidden = torch.ones((c["new"], total[i]), dtype=torch.bool, device=DEV).triu(total[i] - c["new"] + 1).repeat(grp, 1)
            x = torch.bmm(q, torch.cat([pk, ok], 1).transpose(1, 2).contiguous()) * scale
            x[:, :, pk.shape[1]:].masked_fill_(hidden, -math.inf)
            y = torch.bmm(torch.softmax(x, -1), torch.cat([pv, ov], 1)).view(c["kv_heads"], grp, c["new"], -1)
            out[r] = y.permute(2, 0, 1, 3).reshape(c["new"], c["q_heads"], -1)
            lse[r] = torch.logsumexp(x, -1).view(c["kv_heads"], grp, c["new"]).permute(2, 0, 1).reshape(c["new"], -1)
            if c["kind"] == "weigh":
                said = s.lse[r].double().view(c["new"], c["kv_heads"], grp).permute(1, 2, 0).reshape(c["kv_heads"], -1, 1)
                p = torch.exp(x - said).sum(1)
                on_prefix = on_prefix + p[:, :pk.shape[1]]
                note(i, total[i], p[:, pk.shape[1]:], total[i] - c["new"])
        if c["kind"] == "weigh" and c["prefix"]:
            note(m + g, total[m + g], on_prefix, total[m + g])
    return {"out": out, "lse": lse} if c["kind"] == "shared" else {"weight": weight}


def _exact_cut(s, layer, i, n, k, v):
    """What is left of n tokens of every head of request i, in the order in which it is left."""
    c = s.case
    if n <= c["keep"]:
        return k, v
    recent = min(c["recent"], c["keep"])
    first, k, v = c["keep"] - recent, k.clone(), v.clone()
    t = torch.arange(n, device=DEV)
    weight = s.weight[layer][s.table[i, t // c["block"]].long(), :, t % c["block"]].cpu().numpy()      # [tokens, kv_heads]
    for h in range(c["kv_heads"]):
        chosen = set(np.lexsort((np.arange(n - recent), -weight[:n - recent, h].astype(np.float64)))[:first].tolist())
        holes = [t for t in range(first) if t not in chosen]
        order = list(range(first)) + list(range(n - recent, n))
        for hole, filler in zip(holes, sorted(t for t in chosen if t >= first)):
            order[hole] = filler
        at = torch.tensor(order, device=DEV)
        k[h, :c["keep"]], v[h, :c["keep"]] = k[h, at], v[h, at]
    return k[:, :c["keep"]], v[:, :c["keep"]]
