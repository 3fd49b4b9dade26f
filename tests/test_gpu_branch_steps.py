"""Steps of beams behind shared prefixes through PagedCache: choice, fork, positions, append, attention over prefix and own tokens, weights and evictions together,
eager, in a graph and on two streams, against books kept in 64 bits.  Tolerances: those of test_gpu_branch.py."""
import numpy as np
import pytest

import branch_reference as branch
import paged_reference as ref

torch = pytest.importorskip("torch")
from test_gpu_branch import check_select, prefix_of  # noqa: E402
from test_gpu_paged import DEV, check_rope, host, i32, lse_tolerance, randn, tolerance  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(scope="module")
def P():
    import paper_2603_17573_amd as P
    return P


class Run:
    """groups of beams requests each, then a prefix request for every group; the tokens of every request as lists of rows that the cache holds."""

    def __init__(self, P, rng, groups, beams, heads, hd, dtype, layers=2, block=16, prefix=120, vocab=300, max_own=96, n_blocks=None, weights=True):
        self.P, self.rng, self.groups, self.beams, self.heads, self.hd, self.dtype, self.layers = P, rng, groups, beams, heads, hd, dtype, layers
        self.n, self.batch, self.vocab = groups * beams, groups * beams + groups, vocab
        self.c = P.PagedCache(layers, *heads, hd, self.batch, 160, 2 * groups * prefix, n_blocks=n_blocks or 14 * self.batch, block_size=block, max_new=1,
                              weights=weights)
        self.first = i32([beams * g for g in range(groups + 1)])
        self.prefix = i32([self.n + g for g in range(groups)])
        self.c.share(self.first, self.prefix, beams, max_prefix=160, max_own=max_own)
        self.rows = [[[] for _ in range(self.batch)] for _ in range(layers)]      # (k, v), each [kv_heads, d]
        self.gone = np.zeros(self.batch, int)                                      # tokens that were evicted
        self.freq, self.size = ref.frequencies(hd, 10000.0)
        self.score = torch.tensor(-rng.random(self.n), dtype=torch.float32, device=DEV)
        self.done = torch.zeros(self.n, dtype=torch.int32, device=DEV)
        self.length = torch.zeros(self.n, dtype=torch.int32, device=DEV)
        self.parent = torch.arange(self.batch, dtype=torch.int32, device=DEV)
        self.offset = torch.zeros(self.batch, dtype=torch.int32, device=DEV)

    def inputs(self, rows):
        return [[randn(self.rng, (rows, h, self.hd), self.dtype) for h in (self.heads[0], self.heads[1], self.heads[1])] for _ in range(self.layers)]

    def prompts(self, lengths):
        cached = [-1] * self.n + [0] * self.groups
        new = [0] * self.n + list(lengths)
        self.c.begin(i32(cached), i32(new), sum(new))
        for layer, (q, k, v) in enumerate(self.inputs(sum(new))):
            self.c.rotate(q, k)
            self.c.append(layer, k, v)
            lse = torch.empty(q.shape[:2], device=DEV)
            self.c.attend(layer, q, lse=lse)
            if self.c.weights is not None:
                self.c.weigh(layer, q, lse)
            at = 0
            for g, n in enumerate(lengths):
                self.note(layer, self.n + g, host(k)[at:at + n], host(v)[at:at + n])
                at += n
        self.offset[:self.n] = i32(np.repeat(lengths, self.beams))
        torch.cuda.synchronize()

    def note(self, layer, request, k, v):
        self.rows[layer][request] += list(zip(ref.held(k), ref.held(v)))

    def lengths(self):
        return [len(r) for r in self.rows[0]]

    def step(self, cached, q, k, v, logits):
        """The calls of one step; what they return."""
        s = self.P.beam_select(logits, self.beams, self.beams, self.score, self.length, self.done, 3, 0.5, parent=self.parent, stride=self.beams)
        lengths = self.c.fork(self.parent, cached)
        self.c.begin(lengths, self.new, self.n)
        self.c.offset(self.offset)
        outs = []
        for layer in range(self.layers):
            self.c.rotate(q[layer], k[layer])
            self.c.append(layer, k[layer], v[layer])
            lse = torch.empty(q[layer].shape[:2], device=DEV)
            outs.append((self.c.attend_shared(layer, q[layer], lse=lse), lse))
            if self.c.weights is not None:
                self.c.weigh(layer, q[layer], lse, decay=0.9)
        return s, outs

    def check(self, s, outs, q0, k0, q, k, v, logits, before):
        """before: score, length and done that the choice was made from."""
        check_select(s, logits, self.beams, self.beams, before[0], before[1], before[2], 3, 0.5)
        parent = [g * self.beams + int(s["beam"][g, n]) for g in range(self.groups) for n in range(self.beams)]
        assert self.parent[:self.n].tolist() == parent and self.parent[self.n:].tolist() == list(range(self.n, self.batch))
        for layer in range(self.layers):
            self.rows[layer] = [list(self.rows[layer][p]) for p in parent] + self.rows[layer][self.n:]
        position = i32([int(self.offset[i]) + len(self.rows[0][i]) for i in range(self.n)])
        groups = (self.first.tolist(), self.prefix.tolist())
        for layer in range(self.layers):
            check_rope(q0[layer], q[layer], position, self.freq, self.size, "half", False, self.dtype)
            check_rope(k0[layer], k[layer], position, self.freq, self.size, "half", False, self.dtype)
            for i in range(self.n):
                self.note(layer, i, host(k[layer])[i:i + 1], host(v[layer])[i:i + 1])
            out, lse = (host(x) for x in outs[layer])
            parents = prefix_of(groups, self.batch, self.lengths(), 160)
            for i in range(self.n):
                rows = self.rows[layer][parents[i]] + self.rows[layer][i]
                kk, vv = (np.stack([r[j] for r in rows]) for j in (0, 1))
                want, wl, mean, flat, size = ref.attention(host(q[layer])[i:i + 1], kk, vv, [len(rows)], self.hd ** -0.5)
                assert np.all(np.abs(out[i:i + 1] - want) <= tolerance(self.dtype, 2.0 ** -11, 2.0 ** -36, self.hd, len(rows), want, mean, flat, size))
                assert np.all(np.abs(lse[i:i + 1] - wl) <= lse_tolerance(self.hd, len(rows), wl, size))

    def weights_of(self, layer, request):
        c, n = self.c, len(self.rows[layer][request])
        slots = host(c.table)[request].astype(int)[np.arange(n) // c.block_size]
        return host(c.weights[layer])[slots, :, np.arange(n) % c.block_size]           # [tokens, kv_heads]

    def evict(self, keep, recent):
        """Heads keep tokens of their own: a request's rows then hold, head by head, what that head kept."""
        before = [[self.weights_of(layer, i) for i in range(self.batch)] for layer in range(self.layers)]
        lengths = self.c.evict(i32(keep), recent)
        for layer in range(self.layers):
            for i in range(self.batch):
                rows, w = self.rows[layer][i], before[layer][i]
                if not rows:
                    continue
                order = [branch.cut(w[:, h], keep[i], recent) for h in range(self.heads[1])]
                self.rows[layer][i] = [(np.stack([rows[order[h][t]][0][h] for h in range(self.heads[1])]),
                                        np.stack([rows[order[h][t]][1][h] for h in range(self.heads[1])])) for t in range(len(order[0]))]
        assert lengths.tolist()[self.n:] == self.lengths()[self.n:]
        return lengths


def go(r, steps, evictions=()):
    r.new = i32([1] * r.n + [0] * r.groups)
    for step in range(steps):
        logits = randn(r.rng, (r.n, r.vocab), "bf16", spread=False)
        q, k, v = ([x[j] for x in r.inputs(r.n)] for j in range(3))
        q0, k0 = [x.clone() for x in q], [x.clone() for x in k]
        before = (r.score.clone(), r.length.clone(), r.done.clone())
        s, outs = r.step(i32(r.lengths()), q, k, v, logits)
        torch.cuda.synchronize()
        r.check(s, outs, q0, k0, q, k, v, logits, before)
        r.score, r.length, r.done = s["score"].view(-1), s["length"].view(-1), s["done"].view(-1)
        if step in evictions:
            lengths = r.lengths()
            keep = [-1 if i < r.n else max(1, lengths[i] - 20) for i in range(r.batch)]
            r.evict(keep, 9)
        used = {int(x) for b in range(r.batch) for x in host(r.c.table)[b, :int(host(r.c.owned)[b])]}
        free = {int(x) for x in host(r.c.free_ids)[:int(host(r.c.free_count)[0])]}
        assert not used & free and len(used) + len(free) == r.c.n_blocks and len(used) == int(host(r.c.owned).sum())


@pytest.mark.parametrize("dtype,groups,beams,heads,hd,max_own", [("bf16", 2, 4, (4, 2), 64, 96), ("f16", 1, 3, (6, 2), 128, 96), ("bf16", 1, 20, (8, 2), 128, 96),
                                                                 ("f16", 2, 17, (4, 1), 64, 1200), ("bf16", 3, 2, (2, 2), 128, 96)])
def test_beams(P, dtype, groups, beams, heads, hd, max_own):
    rng = np.random.default_rng(beams + hd)
    r = Run(P, rng, groups, beams, heads, hd, dtype, max_own=max_own)
    r.prompts([int(x) for x in rng.integers(40, 120, groups)])
    go(r, 5, evictions=(1, 3))


def test_beams_in_a_graph(P):
    """A step captured once and replayed, with the program's own work between: what it reads is copied into its inputs."""
    rng = np.random.default_rng(11)
    r = Run(P, rng, 2, 17, (4, 1), 64, "bf16", layers=1)
    r.prompts([70, 101])
    r.new = i32([1] * r.n + [0] * r.groups)
    go(r, 1)                                                           # and once before the capture
    q, k, v = ([x[j] for x in r.inputs(r.n)] for j in range(3))
    logits = randn(rng, (r.n, r.vocab), "bf16", spread=False)
    cached = i32(r.lengths())
    r.score, r.length, r.done = r.score.clone(), r.length.clone(), r.done.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            s, outs = r.step(cached, q, k, v, logits)
            lengths = r.c.evict(keep := torch.full((r.batch,), -1, dtype=torch.int32, device=DEV), 5)
    for n in range(5):
        for t in (*q, *k, *v):
            t.copy_(randn(rng, tuple(t.shape), "bf16"))
        logits.copy_(randn(rng, tuple(logits.shape), "bf16", spread=False))
        cached.copy_(i32(r.lengths()))
        q0, k0 = [x.clone() for x in q], [x.clone() for x in k]
        before = (r.score.clone(), r.length.clone(), r.done.clone())
        graph.replay()
        torch.cuda.synchronize()
        r.check(s, outs, q0, k0, q, k, v, logits, before)
        assert lengths.tolist() == r.lengths()
        for a, b in ((r.score, "score"), (r.length, "length"), (r.done, "done")):
            a.copy_(s[b].view(-1))
        assert np.isfinite(torch.randn(1 << 20, device=DEV).sum().item())      # the program's own work between replays
    assert keep.tolist() == [-1] * r.batch


def test_two_runs_on_two_streams(P):
    """Two caches in flight at once give what each gives alone."""
    outs = []
    for together in (False, True):
        runs = [Run(P, np.random.default_rng(s), 1, 16, (8, 2), 128, "bf16", layers=1) for s in (1, 2)]
        streams = [torch.cuda.Stream(), torch.cuda.Stream()] if together else [torch.cuda.current_stream()] * 2
        got, ins = [[], []], []
        for r in runs:
            r.prompts([100])
            r.new = i32([1] * r.n + [0])
            ins.append([(r.inputs(r.n)[0], randn(r.rng, (r.n, r.vocab), "bf16", spread=False)) for _ in range(4)])
        torch.cuda.synchronize()
        cached = [i32([0] * r.n + [100]) for r in runs]
        for n in range(4):
            for j, r in enumerate(runs):
                with torch.cuda.stream(streams[j]):
                    (q, k, v), logits = ins[j][n]
                    s, o = r.step(cached[j], [q], [k], [v], logits)
                    r.score = s["score"].view(-1)
                    cached[j] = r.c.seq_len.clone()
                    got[j] += [o[0][0], o[0][1], s["token"], s["beam"], s["score"]]
        torch.cuda.synchronize()
        outs.append([[t.clone() for t in g] + [r.c.weights.nan_to_num(0).clone()] for g, r in zip(got, runs)])
    for a, b in zip(*outs):
        assert all(torch.equal(x, y) for x, y in zip(a[:-1], b[:-1]))


def test_refusals_of_the_cache(P):
    c = P.PagedCache(1, 4, 2, 64, 4, 200, 300, n_blocks=30, block_size=16)
    q, lse = torch.empty((0, 4, 64), dtype=torch.bfloat16, device=DEV), torch.empty((0, 4), device=DEV)
    with pytest.raises(ValueError, match="without share"):
        c.attend_shared(0, q)
    with pytest.raises(ValueError, match="without weights"):
        c.weigh(0, q, lse)
    with pytest.raises(ValueError, match="without weights"):
        c.evict(i32([1] * 4), 0)
    for bad in (i32([0] * 3), torch.zeros(4, dtype=torch.int64, device=DEV), torch.zeros(4, dtype=torch.int32)):
        for call in (lambda: c.fork(bad, i32([0] * 4)), lambda: c.fork(i32([0] * 4), bad), lambda: c.offset(bad)):
            with pytest.raises(ValueError):
                call()
    with pytest.raises(ValueError):
        c.share(i32([0, 2]), i32([3, 2]), 1)
    with pytest.raises(ValueError, match="invalid groups"):
        c.share(i32([0, 2]), i32([3]), 0)
    c.share(i32([0, 2]), i32([3]), 2)
    w = P.PagedCache(1, 4, 2, 64, 4, 200, 300, n_blocks=30, block_size=16, weights=True)
    with pytest.raises(RuntimeError, match="kv4_evict"):
        w.evict(i32([1] * 4), -1)
    logits, score = torch.zeros((4, 10), device=DEV), torch.zeros(4, device=DEV)
    for kw in (dict(beams=3), dict(beams=0), dict(score=torch.zeros(3, device=DEV)), dict(score=torch.zeros(4, dtype=torch.float64, device=DEV)),
               dict(logits=logits.double()), dict(logits=logits.cpu()), dict(logits=logits.T), dict(parent=i32([0] * 3), stride=2)):
        with pytest.raises(ValueError):
            P.beam_select(**{**dict(logits=logits, beams=2, width=2, score=score), **kw})
    for kw in (dict(width=65), dict(width=0), dict(end_token=3), dict(length_power=0.5), dict(parent=i32([0] * 9), stride=1)):
        with pytest.raises(RuntimeError, match="beam_select"):
            P.beam_select(**{**dict(logits=logits, beams=2, width=2, score=score), **kw})


def test_steps_without_rows(P):
    """Before the first step, after a fork that ends everything, and with empty rows."""
    c = P.PagedCache(1, 4, 2, 64, 3, 200, 300, n_blocks=30, block_size=16, weights=True)
    c.share(i32([0, 2]), i32([2]), 2)
    q, lse = torch.empty((0, 4, 64), dtype=torch.bfloat16, device=DEV), torch.empty((0, 4), device=DEV)
    assert c.attend_shared(0, q, lse=lse).shape == q.shape
    c.weigh(0, q, lse)
    c.offset(i32([1, 2, 3]))
    assert c.evict(i32([1, 2, 3]), 0).tolist() == [-1, -1, -1]
    assert c.fork(i32([-1, 7, -9]), i32([0, 0, 0])).tolist() == [-1, -1, -1]
    c.begin(i32([-1, -1, -1]), i32([0, 0, 0]), 0)
    assert c.attend_shared(0, q).shape == q.shape and int(c.free_count) == 30


def test_steps_of_any_number_of_rows(P):
    """The workspace is made for the largest step; smaller ones are cut otherwise and fit it, whatever the bounds are."""
    rng = np.random.default_rng(4)
    for max_own in (60, 1500):
        for max_rows in (1, 9, 40, 4000):
            c = P.PagedCache(1, 8, 2, 64, 9, 1500, 400, n_blocks=400, block_size=16, max_new=40)
            c.share(i32([0, 8]), i32([8]), max_rows, max_own=max_own)
            size = P.heisd_kv4_shared_attention_workspace_bytes
            most = c._shared[2].numel()
            for n in (0, 1, 2, 7, 8, 15, 16, 17, 64, 399, 400):
                assert size(c.descs[0], 9, n, 8, 40, max_own, c._shared[0]) <= most
    cached, new = [0] * 8 + [0], [0] * 8 + [300]
    c.begin(i32(cached), i32(new), 300)
    k, v = (randn(rng, (300, 2, 64), "bf16") for _ in range(2))
    c.append(0, k, v)
    rows = [[] for _ in range(8)]
    for n in (1, 40, 3, 1):
        c.begin(i32([len(r) for r in rows] + [300]), i32([n] * 8 + [0]), 8 * n)
        q, k2, v2 = (randn(rng, (8 * n, h, 64), "bf16") for h in (8, 2, 2))
        c.append(0, k2, v2)
        out = host(c.attend_shared(0, q))
        hk, hv = ref.held(host(k2)), ref.held(host(v2))
        for i in range(8):
            rows[i] += list(zip(hk[i * n:(i + 1) * n], hv[i * n:(i + 1) * n]))
            kk, vv = (np.concatenate([ref.held(host(x)), np.stack([r[j] for r in rows[i]])]) for j, x in ((0, k), (1, v)))
            seen = [len(kk) - n + j + 1 for j in range(n)]
            want, _, mean, flat, size = ref.attention(host(q)[i * n:(i + 1) * n], kk, vv, seen, 0.125)
            assert np.all(np.abs(out[i * n:(i + 1) * n] - want) <= tolerance("bf16", 2.0 ** -11, 2.0 ** -36, 64, len(kk), want, mean, flat, size))



def test_a_graph_outlives_its_sharing(P):
    """What share() was given and allocated stays with a captured graph, and with what other streams have queued, when it is called again."""
    c = P.PagedCache(1, 8, 2, 64, 9, 1500, 400, n_blocks=400, block_size=16, weights=True)
    rng = np.random.default_rng(5)
    c.begin(i32([0] * 9), i32([0] * 8 + [300]), 300)
    k, v = (randn(rng, (300, 2, 64), "bf16") for _ in range(2))
    c.append(0, k, v)
    c.begin(i32([0] * 8 + [300]), i32([1] * 8 + [0]), 8)
    q, k, v = (randn(rng, (8, h, 64), "bf16") for h in (8, 2, 2))
    c.append(0, k, v)
    c.weights.zero_()

    def share(*edges):
        c.share(i32(edges), i32([8]), 8, max_prefix=300, max_own=1500)

    def run():
        lse = torch.empty(8, 8, device=DEV)
        out = c.attend_shared(0, q, lse=lse)
        c.weigh(0, q, lse, decay=0.0)
        return out, lse

    share(0, 8)
    want = [*run(), c.weights.clone()]
    share(0, 3)
    other = [*run(), c.weights.clone()]
    share(0, 8)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            got = run()
    size = c._shared[2].numel()
    for n in range(3):
        share(0, 3)                                                    # the first one is the graph's alone now
        filled = [torch.full((size,), 255, dtype=torch.uint8, device=DEV) for _ in range(4)] + [i32([7, 7]) for _ in range(40)]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*got, c.weights), want))
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            eager = run()
        share(0, 1)                                                    # while that may still run
        filled += [torch.full((size,), 255, dtype=torch.uint8, device=DEV) for _ in range(2)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*eager, c.weights), other))
    assert not torch.equal(want[0], other[0])


def test_lengths_that_a_call_gave_bound_the_next(P):
    """keep, lengths: the buffer of the last evict() or fork() itself."""
    c = P.PagedCache(1, 4, 2, 64, 3, 64, 100, n_blocks=12, block_size=16, weights=True)
    c.begin(i32([0] * 3), i32([20, 40, 30]), 90)
    k, v = (torch.randn(90, 2, 64, device=DEV).bfloat16() for _ in range(2))
    c.append(0, k, v)
    c.weights.fill_(1.0)
    kept = c.evict(i32([10, -1, 64]), 4)
    assert kept.tolist() == [10, 40, 30]
    c.seq_len.copy_(i32([20, 40, 30]))
    assert c.evict(kept, 4).tolist() == [10, 40, 30]
    kept = c.fork(i32([0, 1, 2]), kept)
    assert c.fork(i32([2, 1, 0]), kept, trim=True).tolist() == [30, 40, 10] and int(c.free_count) == 6
