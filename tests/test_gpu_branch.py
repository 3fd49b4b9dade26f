"""Requests that continue others through the C ABI, against the plain definitions of branch_reference.py and paged_reference.py.

Tolerances.  Whole numbers, copies and evictions are exact.  Beams: a score is a logit, a sum in 64 bits and the logarithm of a sum of exponentials; an
exponential is off by 2^-22, its sum over a thread's 32 values and a wave by 40 additions of 2^-24, the sums of chunks are joined in 64 bits: at most 2^-18
absolutely, and the result is rounded once.  Continuations whose ranks are nearer than that may be in either order, exactly equal ones may not.
Shared attention: that of heisd_kv4_attention over the prefix's and the request's own tokens (test_gpu_paged.py); over a prefix a probability p
may enter the product as one fp16 number, off by 2^-11 p or, below 2^-25 of the largest, by 2^-36 of it, which moves sum(p v) / sum(p) by at most
2^-11 of the weighted mean of |v| and 2^-36 of the sum of |v| over the largest weight's sum.  Weights: a score is off by S = (head_dim + 8)
2^-24 * scale * sum |q_i k_i|, the exponent's argument by 2^-22 of its parts and an exponential by 2^-22; sums of n of them add (n + 32) 2^-24."""
import math

import numpy as np
import pytest

import branch_reference as branch
import paged_reference as ref

torch = pytest.importorskip("torch")
from test_gpu_paged import DEV, DTYPES, Cache, host, i32, lse_tolerance, ok, randn, stream, tolerance  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(scope="module")
def P():
    import paper_2603_17573_amd as P
    return P


# ---- the next beams -----------------------------------------------------------------------------------------------------

def run_select(P, logits, beams, width, score, length=None, done=None, end_token=-1, power=0.0, parent=None, first=0, stride=0):
    groups = logits.shape[0] // beams
    o = {k: torch.full((groups, width), -7, dtype=torch.int32, device=DEV) for k in ("beam", "token")}
    o["score"] = torch.full((groups, width), 7.0, device=DEV)
    if length is not None:
        o["length"] = torch.full((groups, width), -7, dtype=torch.int32, device=DEV)
    if done is not None:
        o["done"] = torch.full((groups, width), -7, dtype=torch.int32, device=DEV)
    d = P.make_beam_desc(logits, beams, width, score, o["score"], o["beam"], o["token"], length, o.get("length"), done, o.get("done"), end_token,
                         power, parent, first, stride)
    n = P.heisd_beam_select_workspace_bytes(groups, beams, width, logits.shape[1])
    ws = torch.full((n,), 255, dtype=torch.uint8, device=DEV)
    ok(P, P.heisd_beam_select(d, ws.data_ptr(), n, stream()))
    torch.cuda.synchronize()
    return o


def check_select(o, logits, beams, width, score, length=None, done=None, end_token=-1, power=0.0):
    x, s = host(logits), host(score)
    ln, dn = (None if t is None else host(t).astype(int) for t in (length, done))
    for g in range(x.shape[0] // beams):
        r = slice(g * beams, (g + 1) * beams)
        want = branch.candidates(x[r], s[r], None if ln is None else ln[r], None if dn is None else dn[r], end_token, power)
        rank = {(c[2], c[3]): c[0] for c in want}
        taken = set()
        for n in range(width):
            beam, token, got = int(o["beam"][g, n]), int(o["token"][g, n]), float(o["score"][g, n])
            if n >= len(want):
                assert (beam, token, got) == (-1, -1, -math.inf)
                assert done is None or int(o["done"][g, n]) == 1
                assert length is None or int(o["length"][g, n]) == 0
                continue
            c = want[n]
            assert (beam, token) in rank and (beam, token) not in taken
            taken.add((beam, token))
            tol = 2.0 ** -18 + 2.0 ** -24 * abs(c[1])
            if (beam, token) != (c[2], c[3]):
                assert rank[beam, token] != c[0] and abs(rank[beam, token] - c[0]) <= 2 * tol, (g, n, beam, token, c)
                c = next(w for w in want if (w[2], w[3]) == (beam, token))
            assert abs(got - c[1]) <= tol
            assert length is None or int(o["length"][g, n]) == c[4]
            assert done is None or int(o["done"][g, n]) == c[5]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("groups,beams,width,vocab", [(1, 1, 1, 1), (1, 4, 4, 256), (3, 2, 5, 7), (2, 8, 8, 32000), (5, 3, 3, 8191), (1, 64, 64, 257),
                                                      (2, 1, 64, 8193), (1, 5, 16, 40001), (1, 2, 4, 131071), (130, 4, 4, 300)])
def test_select(P, dtype, groups, beams, width, vocab):
    rng = np.random.default_rng(vocab + beams)
    logits = randn(rng, (groups * beams, vocab), dtype, spread=False)
    score = torch.tensor(-5 * rng.random(groups * beams), dtype=torch.float32, device=DEV)
    check_select(run_select(P, logits, beams, width, score), logits, beams, width, score)
    length = i32(rng.integers(0, 9, groups * beams))
    done = i32(rng.random(groups * beams) < 0.3)
    args = (beams, width, score, length, done, vocab // 2, 0.7)
    check_select(run_select(P, logits, *args), logits, *args)


def test_select_ties_and_values_that_are_not_finite(P):
    """Equal logits and equal beams: the lowest beam, then the lowest token.  Masked, infinite and missing ones."""
    rng = np.random.default_rng(2)
    for vocab in (50, 9000, 20000):
        x = np.round(rng.standard_normal((8, vocab)), 1)
        x[1] = x[0]
        x[3] = 0.25                                                    # all equal
        x[4, :] = -math.inf
        x[4, [vocab - 1, 17]] = 1.0
        x[5, ::2] = math.nan
        x[6, 3] = math.inf
        x[7] = -math.inf
        score = torch.tensor([-1, -1, -math.inf, -1, -2, -3, -1, math.nan], dtype=torch.float32, device=DEV)
        for dtype in ("f32", "bf16"):
            logits = torch.tensor(x, device=DEV).to(DTYPES[dtype])
            for beams, width in ((8, 8), (8, 64), (4, 20), (1, 9), (2, 33)):
                args = (beams, width, score[:8 // beams * beams])
                check_select(run_select(P, logits, *args), logits, *args)
    logits = torch.zeros((4, 30000), dtype=torch.bfloat16, device=DEV)
    o = run_select(P, logits, 4, 64, torch.tensor([-3.0, -2.0, -2.0, -4.0], device=DEV))
    assert o["token"][0].tolist() == list(range(64)) and o["beam"][0].tolist() == [1] * 64


def test_select_layouts(P):
    """Rows apart, at odd addresses, all at the same place; parents of requests; in place."""
    rng = np.random.default_rng(3)
    for dtype in ("f32", "bf16"):
        wide = randn(rng, (6, 9100), dtype, spread=False)
        score = torch.tensor(-5 * rng.random(6), dtype=torch.float32, device=DEV)
        for off in (0, 1, 3, 8):
            logits = wide[:, off:off + 9001]
            check_select(run_select(P, logits, 3, 3, score), logits, 3, 3, score)
        logits = wide[:1].expand(6, -1)                                # every beam has the same logits
        check_select(run_select(P, logits, 6, 6, score), logits, 6, 6, score)
        base = wide.reshape(-1)[1:1 + 6 * 9001].view(6, 9001)
        check_select(run_select(P, base, 2, 4, score), base, 2, 4, score)
    parent = torch.arange(11, dtype=torch.int32, device=DEV)
    o = run_select(P, wide, 3, 3, score, parent=parent, first=1, stride=5)
    want = list(range(11))
    for g in range(2):
        for n in range(3):
            want[1 + 5 * g + n] = 1 + 5 * g + int(o["beam"][g, n])
    assert parent.tolist() == want
    length, done = i32(rng.integers(0, 9, 6)), i32([0, 1, 0, 0, 0, 1])
    for _ in range(2):
        args = (3, 3, score.clone(), length.clone(), done.clone(), 5, 1.0)
        d = P.make_beam_desc(wide, 3, 3, score, score, o["beam"], o["token"], length, length, done, done, 5, 1.0)
        n = P.heisd_beam_select_workspace_bytes(2, 3, 3, 9100)
        ws = torch.empty(n, dtype=torch.uint8, device=DEV)
        ok(P, P.heisd_beam_select(d, ws.data_ptr(), n, stream()))
        got = dict(o, score=score.view(2, 3), length=length.view(2, 3), done=done.view(2, 3))
        check_select(got, wide, *args)


# ---- requests that continue others ----------------------------------------------------------------------------------------

def books(rng, batch, block, max_blocks, most, spare, dead=0.1):
    length = [int(rng.integers(0, most + 1)) if rng.random() > dead else -1 for _ in range(batch)]
    owned = [min(max_blocks, -(-max(n, 0) // block) + int(rng.integers(0, 3))) for n in length]
    n_blocks = sum(owned) + max(spare, 1)
    ids = rng.permutation(n_blocks)
    table = np.full((batch, max_blocks), -5, np.int64)
    at = 0
    for i, n in enumerate(owned):
        table[i, :n] = ids[at:at + n]
        at += n
    free_ids = np.full(n_blocks, -1, np.int64)
    free_ids[:n_blocks - at] = ids[at:]
    return dict(length=length, owned=owned, table=table, free_ids=free_ids, free_count=min(spare, n_blocks - at), block=block, n_blocks=n_blocks)


def run_reorder(P, s, parent, trim=False):
    b, most = s["table"].shape
    t = {k: i32(s[k]) for k in ("length", "owned", "table", "free_ids")}
    t["parent"], t["free_count"] = i32(parent), i32([s["free_count"]])
    o = {"len_out": i32([-7] * b), "owned_out": i32([-7] * b), "table_out": i32(np.full((b, most), -7)), "copy_from": i32([-7] * b),
         "free_ids": t["free_ids"], "free_count": t["free_count"]}
    d = P.make_reorder_desc(s["block"], s["n_blocks"], t["parent"], t["length"], t["owned"], t["table"], o["len_out"], o["owned_out"],
                            o["table_out"], o["copy_from"], o["free_ids"], t["free_count"], t["free_count"], trim)
    ok(P, P.heisd_paged_reorder(d, stream()))
    torch.cuda.synchronize()
    want = branch.reorder(parent, s["length"], s["owned"], s["table"], s["free_ids"], s["free_count"], s["block"], trim)
    for k in o:
        assert np.array_equal(np.atleast_1d(host(o[k]).astype(np.int64)), np.atleast_1d(np.asarray(want[k]))), k
    return o


@pytest.mark.parametrize("batch,block,max_blocks,most,spare", [(1, 16, 1, 16, 1), (4, 16, 8, 100, 3), (64, 64, 9, 500, 5), (65, 16, 70, 900, 9),
                                                              (256, 32, 5, 150, 40), (257, 1, 30, 30, 5), (1030, 16, 8, 120, 2000), (2500, 16, 3, 40, 30)])
@pytest.mark.parametrize("trim", [False, True])
def test_reorder(P, batch, block, max_blocks, most, spare, trim):
    rng = np.random.default_rng(batch + most)
    s = books(rng, batch, block, max_blocks, most, spare)
    few = rng.integers(0, batch, max(1, batch // 5))
    for parent in (rng.integers(0, batch, batch), np.arange(batch), np.arange(batch)[::-1], rng.choice(few, batch),
                   np.where(rng.random(batch) < 0.3, rng.integers(-3, batch + 3, batch), np.arange(batch)), np.full(batch, -1),
                   np.full(batch, batch - 1), np.array([2 ** 31 - 1] * batch)):
        run_reorder(P, s, [int(x) for x in parent], trim)


def test_reorder_without_blocks_left(P):
    """First come, first served: nobody after the first refusal is served; what does not fit the table ends."""
    rng = np.random.default_rng(8)
    for spare in (0, 1, 2, 5):
        s = books(rng, 9, 16, 4, 64, spare, dead=0)
        s["length"][0], s["length"][4] = 60, 70
        run_reorder(P, s, [0, 0, 0, 3, 4, 4, 0, 3, 8])
        run_reorder(P, s, [0, 0, 1, 1, 0, 4, 4, 3, 8], True)


@pytest.mark.parametrize("head_dim,block,kv_heads,layers", [(64, 16, 1, 1), (128, 64, 3, 2), (64, 128, 2, 3), (128, 16, 8, 1), (128, 512, 2, 2)])
def test_copy(P, head_dim, block, kv_heads, layers):
    """Whole and partial blocks, all layers, weights with them; nothing else is touched."""
    rng = np.random.default_rng(block + head_dim)
    total = [40, 1, 700, 16, 0, 130, 17, 5]
    c = Cache(P, rng, [700] * 8, kv_heads, head_dim, block)
    pools = torch.randint(0, 256, (layers, c.pool.numel()), dtype=torch.uint8, device=DEV)
    weight = torch.randn((layers, c.n_blocks, kv_heads, block), device=DEV)
    source = [-1, 2, -1, 0, 0, 2, 99, 7]
    length = [40, 700, 700, 40, 0, 333, 17, 5]
    c.table[5, 1 if block < 512 else 0] = -3                            # a block that is not there
    c.t_table = i32(c.table)
    descs = [P.make_kv4_desc(p, block, kv_heads, head_dim) for p in pools]
    want_w, want = weight.clone(), []
    cells = pools.view(layers, c.n_blocks, kv_heads, -1)
    before = cells.clone()
    t_len, t_from = i32(length), i32(source)
    batch = P.make_paged_batch(c.t_table, t_len, None, 0)
    ok(P, P.heisd_kv4_copy(descs[0], layers, pools.shape[1], batch, t_from.data_ptr(), weight.data_ptr(), 700, stream()))
    torch.cuda.synchronize()
    changed = set()
    parts = ((0, head_dim // 2), (block * head_dim // 2, head_dim // 2), (block * head_dim, head_dim // 32),
             (block * head_dim + block * head_dim // 32, head_dim // 32))
    for b, f in enumerate(source):
        if not 0 <= f < 8 or f == b:
            continue
        for j in range(-(-length[b] // block)):
            d, s = int(c.table[b, j]), int(c.table[f, j])
            if not (0 <= d < c.n_blocks and 0 <= s < c.n_blocks):
                continue
            changed.add(d)
            used = min(length[b] - j * block, block)
            for at, per in parts:
                n = used // 4 * 4 * per                               # whole fours of tokens: values lie by four
                assert torch.equal(cells[:, d, :, at:at + n], before[:, s, :, at:at + n])
                end = min((used + 15) // 16 * 16, block) * per
                assert torch.equal(cells[:, d, :, at + end:at + block * per], before[:, d, :, at + end:at + block * per])
            want_w[:, d, :, :used] = want_w[:, s, :, :used]
    same = [x for x in range(c.n_blocks) if x not in changed]
    assert torch.equal(cells[:, same], before[:, same]) and torch.equal(weight, want_w)
    for layer in range(layers):                                        # and as tokens
        c.desc, c.t_seq = descs[layer], t_len
        c.cu_seq = np.concatenate([[0], np.cumsum(length)])
        k, v = c.read(P)
        a, b = int(c.cu_seq[1]), int(c.cu_seq[2])
        assert torch.equal(k[a:b].nan_to_num(9), k[b:b + 700].nan_to_num(9)) and torch.equal(v[a:b].nan_to_num(9), v[b:b + 700].nan_to_num(9))


def test_offset(P):
    rng = np.random.default_rng(4)
    for batch in (1, 5, 70, 500):
        new = rng.integers(0, 9, batch)
        cu = np.concatenate([[0], np.cumsum(new)])
        rows = int(cu[-1]) + 3
        position = rng.integers(-2, 1000, rows)
        offset = rng.integers(-20, 5000, batch)
        offset[0] = 2 ** 31 - 1
        t, o = i32(position), i32(offset)
        table = torch.zeros((batch, 1), dtype=torch.int32, device=DEV)
        ok(P, P.heisd_paged_offset(P.make_paged_batch(table, table.view(-1), i32(cu), rows), o.data_ptr(), t.data_ptr(), stream()))
        want = position.astype(np.int64).copy()
        for b in range(batch):
            for r in range(cu[b], cu[b + 1]):
                if want[r] >= 0:
                    want[r] += offset[b]
                    if not 0 <= want[r] < 2 ** 31:
                        want[r] = -1
        assert np.array_equal(host(t).astype(np.int64), want)


# ---- attention over a shared prefix ---------------------------------------------------------------------------------------

def shared(P, c, groups, q, cu_rows, max_q, max_seq, max_rows, max_prefix, scale, lse=True, out=None, workspace=None):
    rows = q.shape[0]
    out = torch.full_like(q, 7.0) if out is None else out
    lse = torch.full(q.shape[:2], 7.0, device=DEV) if lse else None
    first, prefix = i32(groups[0]), i32(groups[1])
    g = P.make_prefix_groups(first, prefix, max_rows, max_prefix) if len(groups[1]) else None
    n = P.heisd_kv4_shared_attention_workspace_bytes(c.desc, len(c.total), rows, q.shape[1], max_q, max_seq, g)
    assert n > 0
    ws = torch.full((n,), 255, dtype=torch.uint8, device=DEV) if workspace is None else workspace
    ok(P, P.heisd_kv4_shared_attention(c.desc, c.batch(P, cu_rows, rows), g, P.head_rows(q), P.head_rows(out),
                                       lse.data_ptr() if lse is not None else None, scale, max_q, max_seq, ws.data_ptr(), n, stream()))
    torch.cuda.synchronize()
    return out, lse


def prefix_of(groups, batch, seq, max_prefix):
    """The prefix of every request, None where it has none."""
    out = [None] * batch
    first, prefix = groups
    for g, p in enumerate(prefix):
        a, b = first[g], first[g + 1]
        if 0 <= a < b <= batch and 0 <= p < batch and not a <= p < b and 0 < seq[p] <= max_prefix:
            for i in range(a, b):
                out[i] = p
    return out


def check_shared(c, groups, q, out, lse, cu_rows, k, v, scale, dtype, max_prefix, seq=None, gone=None, heads=None):
    seq = list(c.total) if seq is None else seq
    q64, out, lse = host(q), host(out), host(lse)
    parents = prefix_of(groups, len(seq), seq, max_prefix)

    def tokens(i, t):
        keep = np.ones(t, bool) if gone is None else ~gone[i][:t]
        return k[c.cu_seq[i]:c.cu_seq[i] + t][keep], v[c.cu_seq[i]:c.cu_seq[i] + t][keep]

    for i, n in enumerate(seq):
        a, b = cu_rows[i], cu_rows[i + 1]
        for r in range(a, b):
            t = min(max(n - (b - a) + (r - a) + 1, 0), max(n, 0))
            kk, vv = tokens(i, t)
            if parents[i] is not None and n >= 0:
                pk, pv = tokens(parents[i], seq[parents[i]])
                kk, vv = np.concatenate([pk, kk]), np.concatenate([pv, vv])
            want, wl, mean, flat, size = ref.attention(q64[r:r + 1], kk, vv, [len(kk)], scale)
            nan = np.isnan(want)
            assert np.array_equal(np.isnan(out[r:r + 1]), nan), (i, r)
            tol = tolerance(dtype, 2.0 ** -11, 2.0 ** -36, q.shape[2], len(kk), want, mean, flat, size)
            # from here on the rows' type rounds to infinity; a number that may be off by tol need do so only where all of [want - tol, want + tol] lies behind it,
            # and may where some of it does (values of 2^70 that cancel: a sum of 0 against 2^33 is within tol = 2^50)
            limit = 65520 if dtype == "f16" else 2.0 ** 128 - 2.0 ** 119
            huge = ~nan & np.isinf(out[r:r + 1])
            assert np.all(huge[~nan & (np.abs(want) - tol >= limit)]) and np.all((np.abs(want) + tol >= limit)[huge])
            assert np.array_equal(out[r:r + 1][huge & (np.abs(want) > tol)], np.copysign(np.inf, want[huge & (np.abs(want) > tol)]))
            nan |= huge
            assert np.all((np.abs(out[r:r + 1] - want) <= tol)[~nan]), (i, r, np.nanmax(np.abs(out[r] - want)))
            fine = np.isfinite(wl)
            assert np.array_equal(lse[r:r + 1][~fine], wl[~fine], equal_nan=True)
            assert np.all(np.abs(lse[r:r + 1][fine] - wl[fine]) <= lse_tolerance(q.shape[2], len(kk), wl, size)[fine])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("own,prefix,new,heads,head_dim,block", [
    ([[1]], [1], 1, (1, 1), 64, 16), ([[7, 3, 5, 1]], [276], 1, (4, 4), 128, 16), ([[20, 9], [40, 1, 130]], [33, 500], 1, (8, 2), 64, 64),
    ([[9] * 20, [17]], [200, 64], 7, (8, 2), 128, 32), ([[30, 31, 29]], [1000], 3, (6, 2), 64, 128), ([[200, 5], [3], [1, 1]], [16, 1, 129], 1, (7, 1), 128, 16),
    ([[2] * 70], [300], 1, (4, 1), 128, 16), ([[300], [5]], [40, 700], 40, (4, 2), 64, 16)])
def test_shared_attention(P, dtype, own, prefix, new, heads, head_dim, block):
    rng = np.random.default_rng(sum(prefix) + head_dim)
    members = [n for g in own for n in g]
    total = members + list(prefix)
    first = np.concatenate([[0], np.cumsum([len(g) for g in own])]).tolist()
    groups = (first, [len(members) + g for g in range(len(own))])
    c = Cache(P, rng, total, heads[1], head_dim, block)
    k, v = (randn(rng, (sum(total), heads[1], head_dim), dtype) for _ in range(2))
    c.write(P, k, v)
    rows = [min(new, n) for n in members] + [0] * len(own)
    cu = np.concatenate([[0], np.cumsum(rows)]).tolist()
    most = max(cu[first[g + 1]] - cu[first[g]] for g in range(len(own)))
    q = randn(rng, (cu[-1], heads[0], head_dim), dtype)
    scale = head_dim ** -0.5
    out, lse = shared(P, c, groups, q, cu, new, max(members), most, max(prefix), scale)
    check_shared(c, groups, q, out, lse, cu, ref.held(host(k)), ref.held(host(v)), scale, dtype, max(prefix))
    again, _ = shared(P, c, groups, q, cu, new, max(members), most, max(prefix), scale, lse=False)
    assert torch.equal(again, out)
    # other bounds cut the work otherwise
    for max_q, max_seq, max_rows, max_prefix in ((1, max(members), 1, max(prefix)), (64, 4096, 1024, 1 << 16)):
        more, lse = shared(P, c, groups, q, cu, max_q, max_seq, max_rows, max_prefix, scale)
        check_shared(c, groups, q, more, lse, cu, ref.held(host(k)), ref.held(host(v)), scale, dtype, max_prefix)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_shared_attention_of_odd_groups(P, dtype):
    """Prefixes that are not there, are one of the group, are empty or too long; requests of no group, left out, without rows or tokens; blocks
    that are missing; padded rows; a prefix for two groups, and one with rows of its own."""
    rng = np.random.default_rng(77)
    total = [20, 3, 40, 16, 5, 33, 70, 9, 8, 150, 60, 1]
    c = Cache(P, rng, total, 2, 64, 16)
    k, v = (randn(rng, (sum(total), 2, 64), "f32") for _ in range(2))
    c.write(P, k, v)
    c.table[9, 2], c.table[2, 0] = -1, c.n_blocks
    c.t_table = i32(c.table)
    gone = [np.zeros(200, bool) for _ in total]
    gone[9][32:48] = True
    gone[2][:16] = True
    seq = list(total)
    seq[1], seq[11] = -1, 0
    c.t_seq = i32(seq)
    new = [1, 2, 3, 0, 5, 1, 1, 2, 1, 2, 0, 3]
    cu = np.concatenate([[0], np.cumsum(new)]).tolist()
    q = randn(rng, (cu[-1] + 2, 4, 64), dtype)
    for groups in (([0, 3, 5, 7, 9], [9, 10, 9, 11]), ([1, 4, 4, 6, 8], [2, 9, 10, 10]), ([0, 2, 9, 12, 12], [10, 12, 3, -1]), ([0, 12], [0]), ([9, 11, 12], [8, 9]),
                   ([0], []), ([3, 2, 4, 15, 20], [10, 10, 10, 10])):
        for max_prefix in (150, 100):
            out, lse = shared(P, c, groups, q, cu, 5, 70, 9, max_prefix, 0.125)
            # request 9 is longer than max_seq: its own rows see nothing, as a prefix it is what max_prefix says
            assert torch.all(out[cu[9]:cu[10]] == 0) and torch.all(torch.isneginf(lse[cu[9]:cu[10]]))
            assert torch.all(out[cu[-1]:] == 7) and torch.all(lse[cu[-1]:] == 7)
            for i in (j for j in range(12) if j != 9):
                only = [cu[i]] * (i + 1) + [cu[i + 1]] * (12 - i)
                check_shared(c, groups, q, out, lse, only, ref.held(host(k)), ref.held(host(v)), 0.125, dtype, max_prefix, seq=seq, gone=gone)
    # row spans that make no sense: nothing is written, nothing read out of range
    out, lse = shared(P, c, ([0, 6, 12], [10, 9]), q, [0, -5, 90, 4, 2, 2 ** 31 - 1, 3, 99, 98, 97, 96, 95, 94], 5, 150, 9, 150, 0.125)
    assert np.all(host(out) == 7)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_shared_attention_with_values_that_are_not_finite(P, dtype):
    """What is not finite in a prefix reaches every row of its group, in its channels; in a request's own tokens the rows that see it."""
    rng = np.random.default_rng(5)
    total = [40, 9, 12, 8, 300, 200]
    c = Cache(P, rng, total, 1, 128, 16)
    k, v = (randn(rng, (sum(total), 1, 128), "f32") for _ in range(2))
    at = np.concatenate([[0], np.cumsum(total)])
    v[at[4] + 123, 0, 70] = math.inf
    v[at[0] + 38, 0, 3] = math.nan
    k[at[5] + 150, 0, 9] = math.nan
    k[at[2] + 11, 0, 9] = math.inf
    c.write(P, k, v)
    new = [4, 1, 3, 2, 0, 0]
    cu = np.concatenate([[0], np.cumsum(new)]).tolist()
    q = randn(rng, (cu[-1], 3, 128), dtype)
    for groups in (([0, 2], [4]), ([0, 2, 4], [4, 5]), ([2, 4], [4])):
        out, lse = shared(P, c, groups, q, cu, 4, 40, 5, 300, 0.1)
        check_shared(c, groups, q, out, lse, cu, ref.held(host(k)), ref.held(host(v)), 0.1, dtype, 300)


def test_shared_attention_like_the_whole_contexts(P):
    """Many requests over more than a wave of groups: as attention over contexts that hold the prefix themselves."""
    rng = np.random.default_rng(9)
    groups, members, heads, hd = 70, 3, (4, 2), 64
    pre, own = [int(x) for x in rng.integers(1, 90, groups)], [int(x) for x in rng.integers(1, 30, groups * members)]
    total = own + pre
    c = Cache(P, rng, total, heads[1], hd, 16)
    k, v = (randn(rng, (sum(total), heads[1], hd), "bf16") for _ in range(2))
    c.write(P, k, v)
    cu = list(range(len(own) + 1)) + [len(own)] * groups
    q = randn(rng, (len(own), heads[0], hd), "bf16")
    g = ([members * i for i in range(groups + 1)], [len(own) + i for i in range(groups)])
    for scale in (0.125, -0.125, 0.0):
        for max_seq, max_rows in ((30, 3), (30, 64), (4000, 64)):      # narrow; wide; wide with own tokens that may be cut
            out, lse = shared(P, c, g, q, cu, 1, max_seq, max_rows, 90, scale)
            check_shared(c, g, q, out, lse, cu, ref.held(host(k)), ref.held(host(v)), scale, "bf16", 90)


WIDE = 1024      # a bound on the rows of a group that makes many columns of it


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("rows", [2, WIDE])
def test_shared_attention_of_values_far_apart(P, dtype, head_dim, rows):
    """Groups of values whose powers of two lie far apart, small ones beside zero, infinities and NaN, in prefixes of many rows: whatever the form is in which they
    enter the products."""
    rng = np.random.default_rng(head_dim)
    total = [9, 5, 40, 40, 40, 40]
    c = Cache(P, rng, total, 1, head_dim, 16)
    at = np.concatenate([[0], np.cumsum(total)])
    for case in range(6):
        k, v = (randn(rng, (sum(total), 1, head_dim), "f32") for _ in range(2))
        if case == 1:
            v[at[2] + 3, 0, :32] *= 2.0 ** 35
            v[at[3] + 20, 0, -20:] *= 2.0 ** -33
        if case == 2:
            v[at[2] + 3, 0, :32] *= 2.0 ** 90
            v[at[2] + 8, 0, :32] *= 2.0 ** -90
            k[at[3] + 7] *= 2.0 ** -50
        if case == 3:
            v[at[2]:at[3], 0, :32] = 0
            v[at[3]:at[4]] *= 2.0 ** -110
            k[at[2]:at[3], 0, 32:] = 0
        if case == 4:
            v[at[2] + 39, 0, 5] = math.inf
            k[at[3] + 39, 0, 5] = math.nan
        if case == 5:
            k[at[2]:at[3]] = math.nan
        c.pool.fill_(255)
        c.write(P, k, v)
        for groups in (([0, 1, 2], [2, 3]), ([0, 2], [4]), ([0, 2], [2])):
            for cu in ([0, 2, 4, 4, 4, 4, 4], [0, 9, 14, 14, 14, 14, 14]):
                q = randn(rng, (cu[-1], 5, head_dim), dtype)
                out, lse = shared(P, c, groups, q, cu, 9, 40, rows, 40, 0.1)
                check_shared(c, groups, q, out, lse, cu, ref.held(host(k)), ref.held(host(v)), 0.1, dtype, 40)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows", [2, WIDE])
def test_shared_attention_of_zeros_and_of_the_largest(P, dtype, rows):
    """Keys or values that are all zero or as large as a cache holds them, with scales down to zero; prefixes end inside a step."""
    rng = np.random.default_rng(rows)
    total = [9, 5, 70, 40]
    c = Cache(P, rng, total, 1, 64, 16)
    cu, groups = [0, 9, 14, 14, 14], ([0, 1, 2], [2, 3])
    for kf, vf in ((0.0, 1.0), (1.0, 0.0), (2.0 ** -120, 1.0), (1.0, 2.0 ** -124), (1.0, 2.0 ** 112), (2.0 ** 60, 2.0 ** 70)):
        k, v = (randn(rng, (sum(total), 1, 64), "f32", spread=False) for _ in range(2))
        k, v = k * kf, v.clamp(-4, 4) * vf
        c.pool.fill_(255)
        c.write(P, k, v)
        q = randn(rng, (14, 5, 64), dtype)
        for scale in (0.0, 0.1 if kf <= 1 else 2.0 ** -62, -1e-30):
            out, lse = shared(P, c, groups, q, cu, 9, 40, rows, 70, scale)
            check_shared(c, groups, q, out, lse, cu, ref.held(host(k)), ref.held(host(v)), scale, dtype, 70)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("max_seq", [100, 3000])
def test_shared_attention_with_other_bounds(P, dtype, max_seq):
    """More rows than max_q and max_rows say, long tokens of their own, blocks that are missing, padded rows, requests left out; more columns than a workgroup has."""
    rng = np.random.default_rng(max_seq)
    total = [70, 100, 9, 0, 30, 2500 if max_seq > 100 else 60, 700, 90, 333]
    new = [40, 3, 9, 0, 30, 2, 0, 20, 0]
    c = Cache(P, rng, total, 2, 64, 16)
    k, v = (randn(rng, (sum(total), 2, 64), "f32") for _ in range(2))
    c.write(P, k, v)
    gone = [np.zeros(2500, bool) for _ in total]
    c.table[6, 3], c.table[6, 40], c.table[1, 0] = -1, c.n_blocks, -5
    gone[6][48:64], gone[6][640:656], gone[1][:16] = True, True, True
    seq = list(total)
    seq[2] = -1
    c.t_table, c.t_seq = i32(c.table), i32(seq)
    cu = np.concatenate([[0], np.cumsum(new)]).tolist()
    q = randn(rng, (cu[-1] + 3, 8, 64), dtype)
    for groups in (([0, 6], [6]), ([0, 2, 5, 8], [6, 8, 6]), ([4, 6, 6], [0, 8])):
        for max_q, max_rows in ((40, 200), (1, 16), (4, 1000)):
            out, lse = shared(P, c, groups, q, cu, max_q, max_seq, max_rows, 700, -0.125)
            check_shared(c, groups, q, out, lse, cu, ref.held(host(k)), ref.held(host(v)), -0.125, dtype, 700, seq=seq, gone=gone)
            assert torch.all(out[cu[-1]:] == 7) and torch.all(lse[cu[-1]:] == 7)
            again, _ = shared(P, c, groups, q, cu, max_q, max_seq, max_rows, 700, -0.125)
            assert torch.equal(out, again)
    for spans in ([0, -5, 90, 4, 2, 2 ** 31 - 1, 3, 9, 8, 7], [0, 50, 10, 20, 30, 31, 32, 33, 34, 35]):      # nothing read or written out of range
        out, lse = shared(P, c, ([0, 6], [6]), q, spans, 40, max_seq, 200, 700, 0.125)
        assert torch.all(out[50 if spans[1] == 50 else 9:] == 7)       # (request 0 has the rows 0 .. 49 in the second, 7 and 8 have none in either)


def test_layouts(P):
    """Queries and outputs in any order of rows and heads."""
    rng = np.random.default_rng(21)
    total = [9, 5, 40, 7, 130]
    c = Cache(P, rng, total, 2, 128, 16)
    k, v = (randn(rng, (sum(total), 2, 128), "bf16") for _ in range(2))
    c.write(P, k, v)
    cu, groups = [0, 2, 4, 10, 12, 12], ([0, 4], [4])
    q = randn(rng, (12, 8, 128), "bf16")
    for rows in (12, 100):
        want, want_lse = shared(P, c, groups, q, cu, 6, 40, rows, 130, 0.1)
        for make in (lambda t: t.transpose(0, 1).contiguous().transpose(0, 1), lambda t: torch.cat([t, t], 2)[..., :128], lambda t: torch.cat([t, t], 1)[:, 8:]):
            x, o = make(q), make(torch.full_like(q, 7.0))
            out, lse = shared(P, c, groups, x, cu, 6, 40, rows, 130, 0.1, out=o)
            assert torch.equal(out, want) and torch.equal(lse, want_lse)
            check_weigh(P, c, groups, x, lse, cu, 0.1, 0.5, ref.held(host(k)), 40, 130)


def test_a_pool_past_32_bits(P):
    """Blocks more than 4 GiB behind the pool's begin: attention, weights, eviction and copies."""
    rng = np.random.default_rng(8)
    total = [70, 60, 500]
    c = Cache(P, rng, total, 8, 128, 64, spare=66000)
    c.table[:, :9] = np.where(c.table[:, :9] >= 0, c.n_blocks - 1 - np.arange(27).reshape(3, 9), -1)
    c.t_table = i32(c.table)
    assert (c.n_blocks - 30) * 8 * 64 * 136 > 1 << 32
    k, v = (randn(rng, (sum(total), 8, 128), "bf16") for _ in range(2))
    c.write(P, k, v)
    cu, groups = [0, 5, 9, 9], ([0, 2], [2])
    q = randn(rng, (9, 16, 128), "bf16")
    for rows in (9, 100):
        out, lse = shared(P, c, groups, q, cu, 5, 70, rows, 500, 0.1)
        check_shared(c, groups, q, out, lse, cu, ref.held(host(k)), ref.held(host(v)), 0.1, "bf16", 500)
    weight = torch.rand((c.n_blocks, 8, 64), device=DEV)
    first, prefix = i32(groups[0]), i32(groups[1])
    ok(P, P.heisd_kv4_weigh(c.desc, c.batch(P, cu, 9), P.make_prefix_groups(first, prefix, 9, 500), P.head_rows(q), lse.data_ptr(), 0.1, 0.0, weight.data_ptr(),
                            weight.data_ptr(), 70, stream()))
    slots = c.slots()[130:]
    w = host(weight[i32(slots // 64).long(), :, i32(slots % 64).long()])
    want, _ = branch.weights(host(q), ref.held(host(k))[130:], 0.1, host(lse), [500] * 9)
    assert np.allclose(w, want, rtol=1e-4, atol=1e-30)
    out_len = i32([-7] * 3)
    t_keep = i32([-1, -1, 200])
    ok(P, P.heisd_kv4_evict(c.desc, 1, 0, P.make_paged_batch(c.t_table, c.t_seq, None, 0), t_keep.data_ptr(), 50, weight.data_ptr(), weight.data_ptr(), out_len.data_ptr(),
                            500, stream()))
    c.t_seq, c.cu_seq = out_len, np.array([0, 70, 130, 330])
    got = host(c.read(P)[0])
    for h in range(8):
        assert np.array_equal(got[130:, h], ref.held(host(k))[130 + np.array(branch.cut(w[:, h], 200, 50)), h])
    t_from = i32([2, -1, -1])
    c.table[0, :4] = np.arange(4)
    c.t_table, c.t_seq = i32(c.table), i32([200, 60, 200])
    ok(P, P.heisd_kv4_copy(c.desc, 1, 0, P.make_paged_batch(c.t_table, c.t_seq, None, 0), t_from.data_ptr(), weight.data_ptr(), 200, stream()))
    c.cu_seq = np.array([0, 200, 260, 460])
    k2, v2 = c.read(P)
    assert torch.equal(k2[:200], k2[260:]) and torch.equal(v2[:200], v2[260:])


# ---- weights of cached tokens -----------------------------------------------------------------------------------------------

def check_weigh(P, c, groups, q, lse, cu, scale, decay, k, max_seq, max_prefix, seq=None, gone=None, in_place=False):
    seq = list(c.total) if seq is None else seq
    shape = (c.n_blocks, c.kv_heads, c.block)
    weight = torch.rand(shape, device=DEV) + 0.1
    before = host(weight)
    out = weight if in_place else torch.full(shape, -7.0, device=DEV)
    want = host(out).copy()
    first, prefix = i32(groups[0]), i32(groups[1])
    rows = [cu[groups[0][g + 1]] - cu[groups[0][g]] for g in range(len(groups[1]))]
    g = P.make_prefix_groups(first, prefix, max(rows + [1]), max_prefix) if len(groups[1]) else None
    ok(P, P.heisd_kv4_weigh(c.desc, c.batch(P, cu, q.shape[0]), g, P.head_rows(q), lse.data_ptr(), scale, decay, weight.data_ptr(), out.data_ptr(),
                            max_seq, stream()))
    torch.cuda.synchronize()
    q64, l64, got = host(q), host(lse), host(out)
    parents = prefix_of(groups, len(seq), seq, max_prefix)
    bound = np.zeros(shape)
    for i, n in enumerate(seq):
        if n <= 0 or n > max(max_seq, max_prefix if len(groups[1]) else 0):
            continue
        kk = k[c.cu_seq[i]:c.cu_seq[i] + n]
        a, b = cu[i], cu[i + 1]
        count = b - a
        total, size = np.zeros((n, c.kv_heads)), 0.0
        rel = 0
        if n <= max_seq and count:
            total, size = branch.weights(q64[a:b], kk, scale, l64[a:b], [n - count + j + 1 for j in range(count)])
            rel = count * q.shape[1]
        for j, p in enumerate(parents):
            if p == i and cu[j + 1] > cu[j]:
                more, s = branch.weights(q64[cu[j]:cu[j + 1]], kk, scale, l64[cu[j]:cu[j + 1]], [n] * (cu[j + 1] - cu[j]))
                total, size, rel = total + more, max(size, s), rel + (cu[j + 1] - cu[j]) * q.shape[1]
        large = np.abs(np.where(np.isfinite(l64), l64, 0)).max() if l64.size else 0.0
        off = np.expm1(2 * ((c.head_dim + 8) * 2.0 ** -24 * size + 2.0 ** -22 * (size + large + 1))) + (rel + 32) * 2.0 ** -24
        for t in range(n):
            block = c.table[i, t // c.block]
            if not 0 <= block < c.n_blocks:
                continue
            old = before[block, :, t % c.block] if t < n - count else 0.0
            want[block, :, t % c.block] = decay * old + total[t]
            bound[block, :, t % c.block] = off * total[t] + 2.0 ** -23 * np.abs(want[block, :, t % c.block]) + 2.0 ** -100
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan)
    assert np.all((np.abs(got - want) <= bound)[~nan]), np.max((np.abs(got - want) - bound)[~nan])
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("total,new,heads,head_dim,block", [
    ([1], [1], (1, 1), 64, 16), ([1, 2, 15, 16, 17, 33], [1] * 6, (4, 2), 128, 16), ([127, 128, 129, 300], [1, 2, 1, 3], (8, 1), 128, 32),
    ([283], [7], (4, 4), 128, 16), ([5, 90, 0], [5, 40, 0], (6, 2), 64, 64), ([600, 3], [0, 2], (5, 1), 64, 128), ([200], [200], (2, 2), 64, 16)])
def test_weigh(P, dtype, total, new, heads, head_dim, block):
    rng = np.random.default_rng(sum(total) + head_dim)
    c = Cache(P, rng, total, heads[1], head_dim, block)
    k, v = (randn(rng, (sum(total), heads[1], head_dim), dtype) for _ in range(2))
    c.write(P, k, v)
    cu = np.concatenate([[0], np.cumsum(new)]).tolist()
    q = randn(rng, (cu[-1], heads[0], head_dim), dtype)
    scale = head_dim ** -0.5
    out, lse = shared(P, c, ([0], []), q, cu, max(new), max(total), 1, 1, scale)
    kk = ref.held(host(k))
    for in_place in (False, True):
        w = check_weigh(P, c, ([0], []), q, lse, cu, scale, 0.9, kk, max(total), 1, in_place=in_place)
    if sum(new) and block == 16 and total == [283]:                    # what the rows give is one per row and head
        fresh = check_weigh(P, c, ([0], []), q, lse, cu, scale, 0.0, kk, max(total), 1)
        slots = c.slots()
        got = host(fresh)[slots // block, :, slots % block].sum(0)
        assert np.allclose(got, 7 * heads[0] // heads[1], rtol=1e-5)
    if len(total) > 2:
        check_weigh(P, c, ([0], []), q, lse, cu, scale, 1.0, kk, sorted(total)[-2], 1)
        lse[0] = -math.inf
        check_weigh(P, c, ([0], []), q, lse, cu, -scale, 1.0, kk, 1 << 14, 1)
    assert not torch.isnan(w.nan_to_num(0)).any()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_weigh_of_shared_prefixes(P, dtype):
    rng = np.random.default_rng(6)
    total = [20, 3, 40, 16, 5, 33, 70, 9, 300, 150]
    c = Cache(P, rng, total, 2, 128, 16)
    k, v = (randn(rng, (sum(total), 2, 128), dtype) for _ in range(2))
    c.write(P, k, v)
    c.table[9, 2] = -1
    c.t_table = i32(c.table)
    seq = list(total)
    seq[1] = -1
    c.t_seq = i32(seq)
    new = [1, 2, 3, 0, 5, 1, 1, 2, 0, 2]
    cu = np.concatenate([[0], np.cumsum(new)]).tolist()
    q = randn(rng, (cu[-1], 6, 128), dtype)
    for groups in (([0, 3, 5, 8], [8, 9, 8]), ([0, 8], [9]), ([2, 8], [0])):
        out, lse = shared(P, c, groups, q, cu, 5, 150, 14, 300, 0.09)
        lse[cu[1]:cu[2]] = -math.inf
        for in_place in (False, True):
            check_weigh(P, c, groups, q, lse, cu, 0.09, 0.75, ref.held(host(k)), 150, 300, seq=seq, in_place=in_place)


def test_weigh_not_finite(P):
    """A key that is not finite has a weight that is not; the others keep theirs."""
    rng = np.random.default_rng(1)
    c = Cache(P, rng, [50, 20], 1, 64, 16)
    k, v = (randn(rng, (70, 1, 64), "f32") for _ in range(2))
    k[13, 0, 5] = math.nan
    c.write(P, k, v)
    q, lse = randn(rng, (5, 2, 64), "bf16"), torch.full((5, 2), 2.0, device=DEV)
    out = check_weigh(P, c, ([0], []), q, lse, [0, 4, 5], 0.1, 1.0, ref.held(host(k)), 50, 1)
    assert int(torch.isnan(out).sum()) == 1


# ---- eviction -------------------------------------------------------------------------------------------------------------------

def check_evict(P, rng, total, keep, recent, kv_heads, head_dim, block, layers, make=None, in_place=False, seq=None, missing=(), max_seq=1 << 20):
    c = Cache(P, rng, total, kv_heads, head_dim, block)
    pools = torch.full((layers, c.pool.numel()), 255, dtype=torch.uint8, device=DEV)
    descs = [P.make_kv4_desc(p, block, kv_heads, head_dim) for p in pools]
    rows = []
    for d in descs:
        c.desc = d
        k, v = (randn(rng, (sum(total), kv_heads, head_dim), "bf16", spread=False) for _ in range(2))
        c.write(P, k, v)
        rows.append([host(x) for x in c.read(P)])
    for i, j in missing:
        c.table[i, j] = -1
    c.t_table = i32(c.table)
    shape = (layers, c.n_blocks, kv_heads, block)
    w = rng.random(shape) if make is None else make(shape)
    weight = torch.tensor(w, dtype=torch.float32, device=DEV)
    w = host(weight)
    out = weight if in_place else torch.full(shape, -7.0, device=DEV)
    seq = list(total) if seq is None else seq
    t_seq, t_keep, t_out = i32(seq), i32(keep), i32([-7] * len(total))
    batch = P.make_paged_batch(c.t_table, t_seq, None, 0)
    ok(P, P.heisd_kv4_evict(descs[0], layers, pools.shape[1], batch, t_keep.data_ptr(), recent, weight.data_ptr(), out.data_ptr(), t_out.data_ptr(), max_seq,
                            stream()))
    torch.cuda.synchronize()
    got_w = host(out)
    want_w = w.copy() if in_place else np.full(shape, -7.0)
    left = []
    for i, n in enumerate(seq):
        whole = 0 <= n <= max_seq and not any(a == i and b * block < n for a, b in missing)
        left.append(keep[i] if whole and 0 <= keep[i] < n else n)
    assert t_out.tolist() == left
    c.t_seq, c.cu_seq = t_out, np.concatenate([[0], np.cumsum(np.maximum(left, 0))])
    for layer in range(layers):
        c.desc = descs[layer]
        k, v = (host(x) for x in c.read(P))
        at = np.concatenate([[0], np.cumsum(total)])
        for i, n in enumerate(seq):
            if n < 0 or any(a == i for a, _ in missing) or n > max_seq:
                continue
            for h in range(kv_heads):
                t = np.arange(n)
                mine = w[layer, c.table[i, t // block], h, t % block]
                order = branch.cut(mine, keep[i], recent)[:left[i]]
                for was, now in zip(rows[layer], (k, v)):
                    assert np.array_equal(now[c.cu_seq[i]:c.cu_seq[i] + left[i], h], was[at[i] + np.array(order, int), h]), (layer, i, h)
                t = np.arange(left[i])
                want_w[layer, c.table[i, t // block], h, t % block] = mine[order] if left[i] else 0
    if in_place:                                                       # behind what is left the weights may be anything
        for i, n in enumerate(seq):
            t = np.arange(max(left[i], 0), max(n, 0))
            ok_t = t[c.table[i, t // block] >= 0]
            got_w[:, c.table[i, ok_t // block], :, ok_t % block] = want_w[:, c.table[i, ok_t // block], :, ok_t % block]
    assert np.array_equal(got_w, want_w, equal_nan=True)


@pytest.mark.parametrize("head_dim,block,kv_heads,layers", [(64, 16, 1, 1), (128, 64, 2, 2), (128, 16, 3, 1), (64, 128, 2, 2)])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("max_seq", [1100, 8192, 16384, 1 << 20])           # eight keys held by a thread, sixteen, none
def test_evict(P, head_dim, block, kv_heads, layers, in_place, max_seq):
    rng = np.random.default_rng(head_dim + block)
    total = [1, 5, 40, 200, 1100, 64, 0, 333, 90]
    for keep, recent in (([0, 2, 40, 100, 1000, 65, 0, 1, 0], 0), ([1, 4, 39, 199, 40, 63, -1, 300, 17], 16), ([0, 5, 20, 30, 600, 64, 3, 10, 89], 1000),
                         ([-1, 3, -1, 130, 1099, 32, 0, 332, 45], 33)):
        check_evict(P, rng, total, keep, recent, kv_heads, head_dim, block, layers, in_place=in_place, max_seq=max_seq)


def test_evict_many(P):
    """Long contexts, cut by much and by little: the lists of holes and of what fills them take several rounds."""
    rng = np.random.default_rng(3)
    total = [20000, 9001, 16384, 8192]
    for keep, recent in (([10000, 100, 16000, 8000], 64), ([1, 9000, 8192, 2049], 0), ([19999, 4500, 300, 8191], 5000)):
        check_evict(P, rng, total, keep, recent, 1, 64, 64, 1)
    total = [16384, 8193, 8192, 15000]
    for keep, recent in (([8192, 100, 8000, 14999], 64), ([1, 8192, 4096, 7500], 0), ([16383, 4500, 300, 2], 5000)):
        check_evict(P, rng, total, keep, recent, 1, 64, 64, 1, max_seq=16384)
    for keep, recent in (([4096, 100, 8000, 8191], 64), ([1, 8000, 4097, 7500], 0), ([8191, 4500, 300, 2], 5000)):
        check_evict(P, rng, [8192, 8001, 8192, 8192], keep, recent, 2, 128, 32, 1, max_seq=8192, in_place=True)


def test_evict_of_weights_that_are_equal_or_not_numbers(P):
    rng = np.random.default_rng(4)
    total, keep = [300, 2500, 70, 33], [100, 1200, 69, 5]

    def some(values):
        return lambda shape: np.asarray(values)[rng.integers(0, len(values), shape)]
    for values in ([0.0], [0.0, -0.0], [1.0, 2.0], [math.nan], [math.nan, 0.0, 1.0], [-math.inf, math.inf, 3.0, -2.0], [1e-45, 0.0, -1e-45]):
        for in_place in (False, True):
            for max_seq in (2500, 1 << 20):
                check_evict(P, rng, total, keep, 7, 2, 64, 16, 1, make=some(values), in_place=in_place, max_seq=max_seq)


def test_evict_leaves_others_as_they_are(P):
    """Requests left out, with missing blocks or longer than max_seq."""
    rng = np.random.default_rng(5)
    check_evict(P, rng, [100, 90, 300, 50], [50, 40, 20, 10], 8, 2, 64, 16, 2, seq=[100, -1, 300, 50], max_seq=200)
    check_evict(P, rng, [100, 90, 300, 50], [50, 40, 20, 10], 8, 1, 128, 16, 1, missing=[(1, 3), (2, 18)], in_place=True)
