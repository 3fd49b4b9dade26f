"""Requests that continue others where the calls meet each other: groups that describe nothing beside those that do, evictions between other calls, bounds that
differ, the exactness of attention over prefixes of many rows.  Tolerances: those of test_gpu_branch.py, except where a test derives its own."""
import math

import numpy as np
import pytest

import branch_reference as branch
import paged_reference as ref

torch = pytest.importorskip("torch")
from test_gpu_branch import WIDE, check_select, check_shared, check_weigh, prefix_of, run_select, shared  # noqa: E402
from test_gpu_paged import DEV, Cache, host, i32, ok, randn, stream, tolerance  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(scope="module")
def P():
    import paper_2603_17573_amd as P
    return P


# ---- attention over a shared prefix ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("rows,heads", [(12, (4, 2)), (WIDE, (4, 2)), (16, (16, 2))])
@pytest.mark.parametrize("apart", [False, True])
def test_probabilities_are_two_terms_whatever_the_form(P, dtype, head_dim, rows, heads, apart):
    """As exact over a prefix of many rows as over a request's own tokens.  A probability is a bf16 and a bf16 remainder (off by 2^-16 of itself) or an fp16 and an fp16
    remainder (2^-21, or, where its fp16 has few bits, 2^-36 of the largest).  Few tokens and small scores, so that neither an average nor the scores hide
    what a probability is off by: one term alone (2^-11) is too far off.  apart: values whose powers of two lie too far apart for fp16."""
    rng = np.random.default_rng(head_dim + rows)
    total = [3, 3, 4, 5, 3, 20]
    c = Cache(P, rng, total, heads[1], head_dim, 16)
    k, v = (randn(rng, (sum(total), heads[1], head_dim), dtype) for _ in range(2))
    if apart:
        at = np.concatenate([[0], np.cumsum(total)])
        v, k = v.float(), k.float()
        v[at[4] + 2, :, :32] *= 2.0 ** -60
        v[at[5] + 8, :, :32] *= 2.0 ** -60
    c.write(P, k, v)
    new = [3, 3, 2, 4, 0, 0]
    cu, groups = np.concatenate([[0], np.cumsum(new)]).tolist(), ([0, 2, 4], [4, 5])
    q = randn(rng, (cu[-1], heads[0], head_dim), dtype)
    scale = 2.0 / head_dim
    out, lse = shared(P, c, groups, q, cu, 4, 5, rows, 20, scale)
    hk, hv, hq, out = ref.held(host(k)), ref.held(host(v)), host(q), host(out)
    parents = prefix_of(groups, 6, total, 20)
    for i in range(4):
        kk, vv = (np.concatenate([x[c.cu_seq[j]:c.cu_seq[j + 1]] for j in (parents[i], i)]) for x in (hk, hv))
        seen = [len(kk) - new[i] + j + 1 for j in range(new[i])]
        want, _, mean, flat, size = ref.attention(hq[cu[i]:cu[i + 1]], kk, vv, seen, scale)
        over = np.abs(out[cu[i]:cu[i + 1]] - want) - tolerance(dtype, 2.0 ** -16, 2.0 ** -36, head_dim, len(kk), want, mean, flat, size)
        assert over.max() <= 0, (i, float(over.max()), np.argwhere(over > 0)[:4].tolist())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("max_own,max_rows", [(40, 9), (3000, 9), (40, WIDE), (3000, WIDE)])
def test_groups_that_describe_nothing_hide_no_others(P, dtype, max_own, max_rows):
    """Spans that leave the batch, of prefixes that are not there, are empty, too long or one of the group, in front of spans that describe something, in every form; and the
    weights count the same rows."""
    rng = np.random.default_rng(12)
    total = [20, 3, 40, 16, 5, 33, 30, 9, 8, 31, 60, 0]
    c = Cache(P, rng, total, 2, 64, 16)
    k, v = (randn(rng, (sum(total), 2, 64), "f32") for _ in range(2))
    c.write(P, k, v)
    new = [1, 2, 3, 1, 5, 1, 1, 2, 1, 2, 0, 0]
    cu = np.concatenate([[0], np.cumsum(new)]).tolist()
    q = randn(rng, (cu[-1], 4, 64), dtype)
    for groups in (([0, 20, 2, 4], [10, 10, 10]), ([0, 8, 2, 4], [-1, 10, 10]), ([-1, 10, 2, 4], [10, 10, 10]), ([0, 8, 2, 4, 9], [11, 10, 10, 9]),
                   ([0, 9, 2, 4], [8, 10, 9]), ([0, 9, 1, 9], [12, 0, 10]), ([0, 9] * 40 + [3, 5], [-1] * 80 + [10])):
        out, lse = shared(P, c, groups, q, cu, 5, max_own, max_rows, 60, 0.125)
        check_shared(c, groups, q, out, lse, cu, ref.held(host(k)), ref.held(host(v)), 0.125, dtype, 60)
        if max(groups[0]) <= 12:
            check_weigh(P, c, groups, q, lse, cu, 0.125, 0.5, ref.held(host(k)), max_own, 60)
    groups = ([0, 9, 2, 4], [9, 10, 9])                                # prefix 9 has 31 tokens: too long here
    out, lse = shared(P, c, groups, q, cu, 5, max_own, max_rows, 30, 0.125)
    check_shared(c, groups, q, out, lse, cu, ref.held(host(k)), ref.held(host(v)), 0.125, dtype, 30)
    groups = ([0, 9, 2, 4], [10, 10, 9])                               # 10 has 60, 9 has 31
    out, lse = shared(P, c, groups, q, cu, 5, max_own, max_rows, 31, 0.125)
    check_shared(c, groups, q, out, lse, cu, ref.held(host(k)), ref.held(host(v)), 0.125, dtype, 31)


# ---- evictions between other calls of a cache -----------------------------------------------------------------------------

class Rows:
    """A cache of one layer and what its requests' cells hold, as lists of (k, v) with what each head kept."""

    def __init__(self, P, rng, lengths, **more):
        self.c = P.PagedCache(1, 4, 2, 64, len(lengths), 200, 300, block_size=16, weights=True, **more)
        self.rng, self.rows, self.batch = rng, [[] for _ in lengths], len(lengths)
        self.step([0] * self.batch, lengths)

    def step(self, cached, new, takes=None):
        """Appends rows, weighs and attends; checks the attention against what is held.  takes: the requests that the step takes (all)."""
        n = sum(new)
        self.c.begin(cached if torch.is_tensor(cached) else i32(cached), i32(new), n)
        q, k, v = (randn(self.rng, (n, h, 64), "bf16") for h in (4, 2, 2))
        self.c.append(0, k, v)
        lse = torch.empty((n, 4), device=DEV)
        out = self.c.attend(0, q, lse=lse)
        self.c.weigh(0, q, lse)
        hk, hv, hq, out, at = ref.held(host(k)), ref.held(host(v)), host(q), host(out), 0
        for i, m in enumerate(new):
            if takes is None or i in takes:
                self.rows[i] += list(zip(hk[at:at + m], hv[at:at + m]))
                if m:
                    kk, vv = (np.stack([r[j] for r in self.rows[i]]) for j in (0, 1))
                    want, _, mean, flat, size = ref.attention(hq[at:at + m], kk, vv, [len(kk) - m + j + 1 for j in range(m)], 0.125)
                    assert np.all(np.abs(out[at:at + m] - want) <= tolerance("bf16", 2.0 ** -16, 0.0, 64, len(kk), want, mean, flat, size)), i
            else:
                assert not out[at:at + m].any()
            at += m

    def evict(self, keep, recent):
        table, weights = host(self.c.table).astype(int), host(self.c.weights[0])
        lengths = self.c.evict(i32(keep), recent)
        for i, rows in enumerate(self.rows):
            t = np.arange(len(rows))
            w = weights[table[i, t // 16], :, t % 16]
            order = [branch.cut(w[:, h], keep[i], recent) for h in range(2)]
            self.rows[i] = [tuple(np.stack([rows[order[h][t]][j][h] for h in range(2)]) for j in (0, 1)) for t in range(len(order[0]))]
        assert lengths.tolist() == [len(r) for r in self.rows]
        return lengths


def test_eviction_between_a_fork_and_a_step(P):
    """What is cut is what fork() left, and nothing is lost."""
    r = Rows(P, np.random.default_rng(1), [20, 70, 33], n_blocks=30)
    length = r.c.fork(i32([0, 1, 1]), i32([20, 70, 33]))
    assert length.tolist() == [20, 70, 70]
    r.rows[2] = list(r.rows[1])
    length = r.evict([10, 30, -1], 8)
    length = r.evict([10, 30, 40], 8)                                  # and again
    length = r.c.fork(i32([0, 1, 2]), length, trim=True)
    assert length.tolist() == [10, 30, 40] and int(r.c.free_count) == 30 - 1 - 2 - 3
    r.step(length, [1, 2, 1])
    assert r.c.fork(i32([-1, 1, 2]), r.c.seq_len).tolist() == [-1, 32, 41]
    assert r.c.evict(i32([5, 5, 5]), 1).tolist() == [-1, 5, 5]


def test_eviction_makes_room_for_a_request_that_a_step_left_out(P):
    """A request that the plan has no blocks for keeps its tokens; evict() cuts it as it is cached."""
    r = Rows(P, np.random.default_rng(2), [64, 64, 48], n_blocks=12)
    r.step([64, 64, 48], [1, 1, 1], takes=[0])                          # one block is left
    assert r.c.seq_len.tolist() == [65, -1, -1]
    length = r.evict([32, 40, -1], 8)
    assert length.tolist() == [32, 40, 48]
    length = r.c.fork(i32([0, 1, 2]), length, trim=True)
    assert int(r.c.free_count) == 12 - 2 - 3 - 3
    r.step(length, [3, 1, 1])
    assert r.c.seq_len.tolist() == [35, 41, 49]


def test_eviction_after_a_step_that_ended_a_request(P):
    """A finished request stays finished; the others' rows go on being attended to in the same step."""
    r = Rows(P, np.random.default_rng(3), [40, 50, 30], n_blocks=30)
    r.rows[1] = []
    r.step([40, -1, 30], [1, 0, 1])
    assert r.c.evict(i32([41, 9, 20]), 4).tolist() == [41, -1, 20] and r.c.seq_len.tolist() == [41, -1, 20]
    assert r.c.evict(i32([40, 9, 20]), 4).tolist() == [40, -1, 20]


def test_a_step_s_lengths_may_change_after_it(P):
    """begin() does not go on reading the lengths that it was given."""
    r = Rows(P, np.random.default_rng(4), [64, 64, 48], n_blocks=12)
    cached = i32([64, 64, 48])
    r.step(cached, [1, 1, 1], takes=[0])
    cached.fill_(3)
    length = r.evict([32, 40, -1], 8)
    assert length.tolist() == [32, 40, 48]
    r.c.begin(r.c.fork(i32([0, 1, 2]), length), i32([0, 0, 0]), 0)
    r.step(r.c.seq_len, [50, 1, 1], takes=[1])                          # and may be what the step before gave; all blocks are owned
    assert r.c.seq_len.tolist() == [-1, 41, -1]
    assert r.evict([-1, -1, -1], 0).tolist() == [32, 41, 48]


# ---- weights -----------------------------------------------------------------------------------------------------------------

def test_weights_of_requests_longer_than_the_bounds_of_sharing(P):
    """attend() goes as far as the cache, and so do the weights of its rows, whatever share() was told of those that share."""
    rng = np.random.default_rng(5)
    c = P.PagedCache(1, 4, 2, 64, 4, 200, 300, n_blocks=40, block_size=16, weights=True)
    first, prefix = i32([1, 2]), i32([3])
    c.share(first, prefix, 4, max_prefix=64, max_own=16)
    rows = [[] for _ in range(4)]
    for step, (cached, new) in enumerate((([0, -1, 0, 0], [100, 0, 30, 40]), ([100, -1, 30, 40], [2, 0, 1, 0]))):
        c.begin(i32(cached), i32(new), sum(new))
        q, k, v = (randn(rng, (sum(new), h, 64), "bf16") for h in (4, 2, 2))
        c.append(0, k, v)
        if step == 0:
            c.weights.fill_(math.nan)                                  # new tokens have no weight before
        lse = torch.empty((sum(new), 4), device=DEV)
        c.attend(0, q, lse=lse)
        before = host(c.weights[0])
        c.weigh(0, q, lse, decay=0.5)
        got, table, at, hk = host(c.weights[0]), host(c.table).astype(int), 0, ref.held(host(k))
        for i, m in enumerate(new):
            rows[i] += list(hk[at:at + m])
            n = len(rows[i])
            if n:
                t = np.arange(n)
                slot = (table[i, t // 16], slice(None), t % 16)
                want, size = branch.weights(host(q)[at:at + m], np.stack(rows[i]), 0.125, host(lse)[at:at + m], [n - m + j + 1 for j in range(m)])
                old = np.where((t < n - m)[:, None], before[slot], 0.0)
                large = np.abs(host(lse)).max()
                off = np.expm1(2 * (72 * 2.0 ** -24 * size + 2.0 ** -22 * (size + large + 1))) + (4 * m + 32) * 2.0 ** -24
                assert np.all(np.abs(got[slot] - (want + 0.5 * old)) <= off * want + 2.0 ** -23 * (want + 0.5 * old) + 2.0 ** -100), (step, i)
            at += m


def test_weights_at_any_address(P):
    """Weights that begin at any float: eviction moves them as it moves aligned ones."""
    rng = np.random.default_rng(6)
    total, keep = [300, 90, 40], [100, 90, 7]
    c = Cache(P, rng, total, 2, 64, 16)
    k, v = (randn(rng, (sum(total), 2, 64), "bf16") for _ in range(2))
    shape = (c.n_blocks, 2, 16)
    w = torch.rand(shape, device=DEV)
    got = []
    for off in (0, 1, 2, 3):
        c.write(P, k, v)
        held = torch.full((2, w.numel() + 4), -7.0, device=DEV)
        w_in, w_out = (x[off:off + w.numel()].view(shape) for x in held)
        w_in.copy_(w)
        c.t_seq = i32(total)
        out, t_keep = i32([-7] * 3), i32(keep)
        ok(P, P.heisd_kv4_evict(c.desc, 1, 0, P.make_paged_batch(c.t_table, c.t_seq, None, 0), t_keep.data_ptr(), 20, w_in.data_ptr(), w_out.data_ptr(),
                                out.data_ptr(), 300, stream()))
        torch.cuda.synchronize()
        assert out.tolist() == [100, 90, 7] and held[:, :off].eq(-7).all() and held[:, off + w.numel():].eq(-7).all()
        got.append((c.pool.clone(), w_out.clone()))
    assert all(torch.equal(a, b) for x in got[1:] for a, b in zip(x, got[0]))


# ---- copies ------------------------------------------------------------------------------------------------------------------

def test_copies_end_where_they_are_told_to(P):
    """Of requests longer than max_seq the tokens before it are copied; the weights of those behind stay."""
    rng = np.random.default_rng(7)
    c = Cache(P, rng, [60, 60], 2, 64, 64)
    k, v = (randn(rng, (120, 2, 64), "bf16") for _ in range(2))
    c.write(P, k, v)
    weight = torch.rand((c.n_blocks, 2, 64), device=DEV)
    want, source = host(weight), i32([-1, 0])
    for most in (1, 37, 59):
        ok(P, P.heisd_kv4_copy(c.desc, 1, 0, P.make_paged_batch(c.t_table, c.t_seq, None, 0), source.data_ptr(), weight.data_ptr(), most, stream()))
        got = [host(x) for x in c.read(P)]
        want[c.table[1, 0], :, :most] = want[c.table[0, 0], :, :most]
        assert np.array_equal(host(weight), want)
        for x, y in zip(got, (k, v)):
            last = -(-most // 16) * 16                                 # whole tiles of 16 tokens
            held = ref.held(host(y))
            assert np.array_equal(x[60:60 + min(last, 60)], held[:min(last, 60)]) and np.array_equal(x[60 + last:], held[60 + last:])


# ---- the next beams ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_workspaces_hold_every_dtype(P, dtype):
    """A workspace is as large as its function says for any dtype and any number of rows and tokens."""
    rng = np.random.default_rng(8)
    for beams, vocab in ((64, 2044), (64, 2042), (11, 4092), (64, 4097), (64, 8188), (3, 6139), (50, 6138)):
        logits = randn(rng, (beams, vocab), dtype, spread=False)
        score = torch.tensor(-5 * rng.random(beams), dtype=torch.float32, device=DEV)
        check_select(run_select(P, logits, beams, 5, score), logits, beams, 5, score)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("beams,vocab", [(5, 4095), (5, 4096), (5, 4097), (1, 524280)])
def test_select_where_the_forms_meet_and_end(P, dtype, beams, vocab):
    """The largest vocabulary of one launch, the smallest of two, the largest of all, at addresses that cut the first and last segments."""
    rng = np.random.default_rng(vocab)
    whole = randn(rng, (beams * vocab + 16,), dtype, spread=False)
    score = torch.tensor(-5 * rng.random(beams), dtype=torch.float32, device=DEV)
    for off in (0, 1, 3, 7):
        logits = whole[off:off + beams * vocab].view(beams, vocab)
        logits[0, 0] = logits[-1, -1] = 9.0                            # the first and the last token of the rows are among the best
        check_select(run_select(P, logits, beams, 8, score), logits, beams, 8, score)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [51, 257, 4001, 4095, 8191, 32001, 131071])
def test_beams_that_are_equal_are_equal_wherever_their_logits_lie(P, dtype, vocab):
    """Copies of one beam (a first step, say) in rows of odd length, and at odd addresses: the lowest beam first, in each of its tokens."""
    rng = np.random.default_rng(vocab)
    for _ in range(4):
        one = randn(rng, (vocab,), dtype, spread=False)
        whole = torch.empty(9 * (vocab + 3) + 1, dtype=one.dtype, device=DEV)
        logits = whole[1:].view(9, vocab + 3)[:, :vocab]
        logits.copy_(one.expand(9, -1))
        o = run_select(P, logits, 9, 27, torch.full((9,), -1.5, device=DEV))
        best = sorted(range(vocab), key=lambda v, x=host(one): (-x[v], v))[:3]
        rank = host(one)[best]
        want = [(b, v) for x in dict.fromkeys(rank) for b in range(9) for v in (t for t, r in zip(best, rank) if r == x)]
        if len(set(host(one)[sorted(range(vocab), key=lambda v, x=host(one): -x[v])[:4]])) == 4:
            assert list(zip(o["beam"][0].tolist(), o["token"][0].tolist())) == want
        assert all(len(set(o["score"][0][o["token"][0] == v].tolist())) == 1 for v in best)


def test_lengths_whose_power_ends(P):
    """A power of a length that passes 64 bits leaves every continuation its place."""
    logits = torch.tensor([[1.0], [2.0], [3.0]], device=DEV)
    score, length, done = torch.tensor([0.0, -1.0, 0.0], device=DEV), i32([2000, 3, 3000]), i32([0, 0, 1])
    for power in (-200.0, 200.0, -1e9, 1e9):
        o = run_select(P, logits, 3, 3, score, length, done, 0, power)
        assert sorted(o["beam"][0].tolist()) == [0, 1, 2] and o["token"][0].tolist() == [0, 0, 0], power
        assert sorted(o["score"][0].tolist()) == [-1.0, 0.0, 0.0] and sorted(o["length"][0].tolist()) == [4, 2001, 3000]


# ---- two caches at once --------------------------------------------------------------------------------------------------------

def test_weights_of_two_runs_on_two_streams(P):
    """Weights that two caches in flight at once add up and copy are those that each has alone."""
    from test_gpu_branch_steps import Run
    found = []
    for together in (False, True):
        runs = [Run(P, np.random.default_rng(s), 1, 16, (8, 2), 128, "bf16", layers=2) for s in (1, 2)]
        streams = [torch.cuda.Stream(), torch.cuda.Stream()] if together else [torch.cuda.current_stream()] * 2
        ins = []
        for r in runs:
            r.c.weights.zero_()
            r.prompts([100])
            r.new = i32([1] * r.n + [0])
            ins.append([(r.inputs(r.n), randn(r.rng, (r.n, r.vocab), "bf16", spread=False)) for _ in range(6)])
        cached = [i32([0] * r.n + [100]) for r in runs]
        torch.cuda.synchronize()
        for n in range(6):
            for j, r in enumerate(runs):
                with torch.cuda.stream(streams[j]):
                    x, logits = ins[j][n]
                    s, _ = r.step(cached[j], *([y[m] for y in x] for m in range(3)), logits)
                    r.score = s["score"].view(-1)
                    cached[j] = r.c.seq_len.clone()
        torch.cuda.synchronize()
        found.append([(r.c.weights.clone(), r.c.table.clone()) for r in runs])
    for alone, both in zip(*found):
        assert float(alone[0].sum()) > 0 and all(torch.equal(a, b) for a, b in zip(alone, both))
