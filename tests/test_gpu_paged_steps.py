"""The operators on paged requests together, as a decoder calls them: prompts, chunks, drafts with rejections, requests that end and
requests that take their place; the same steps captured into a HIP graph; other streams; two caches at once."""
import math

import numpy as np
import pytest

import paged_reference as ref
from test_gpu_paged import check_attend_rows, check_prompt, host, i32, randn

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(scope="module")
def P():
    import paper_2603_17573_amd as P
    return P


class Book:
    """What every request should have cached, kept by hand: rows as they are held."""

    def __init__(self, batch, layers):
        self.k = [[[] for _ in range(batch)] for _ in range(layers)]
        self.v = [[[] for _ in range(batch)] for _ in range(layers)]

    def add(self, layer, b, at, k, v):
        for rows, x in ((self.k[layer], k), (self.v[layer], v)):
            rows[b] = rows[b][:at] + list(ref.held(x))


def step_inputs(rng, rows, heads, kv_heads, hd, dtype):
    return randn(rng, (rows, heads, hd), dtype), randn(rng, (rows, kv_heads, hd), dtype), randn(rng, (rows, kv_heads, hd), dtype)


def run_step(c, layer, q, k, v, how, total=0):
    c.rotate(q, k)
    c.append(layer, k, v)
    if how == "prompt":
        return c.prompt(q, k, v)
    return c.chunk(layer, q, total) if how == "chunk" else c.attend(layer, q)


def check_step(book, layer, cached, new, q0, k0, q, k, v, out, freq, size, dtype, how):
    """q0, k0: before the rotation; q, k: after it."""
    at = 0
    for b, (p, n) in enumerate(zip(cached, new)):
        if p < 0 or n == 0:
            at += max(n, 0)
            continue
        rows = slice(at, at + n)
        pos = np.arange(p, p + n)
        for x0, x in ((q0, q), (k0, k)):
            want = ref.rope(host(x0)[rows], pos, freq, size, "half", False)
            big = np.abs(host(x0)[rows]).max() * 2 * size
            assert np.abs(host(x)[rows] - want).max() <= ref.half_step(dtype) * big + 2.0 ** -20 * big
        book.add(layer, b, p, host(k)[rows], host(v)[rows])
        if how == "prompt":
            check_prompt(q[rows], k[rows], v[rows], out[rows], None, [0, n], [0, n], q.shape[2] ** -0.5, True, dtype)
        else:
            check_attend_rows(host(q)[rows], host(out)[rows], np.array(book.k[layer][b]), np.array(book.v[layer][b]), q.shape[2] ** -0.5, dtype,
                              chunk=how == "chunk")
        at += n


@pytest.mark.parametrize("dtype,heads,hd,block", [("bf16", (4, 2), 128, 16), ("f16", (6, 2), 64, 32)])
def test_serving(P, dtype, heads, hd, block):
    rng = np.random.default_rng(7)
    batch, layers = 5, 2
    rope = P.make_rope_desc(hd, 500000.0, "parts", 4.0, 64)
    freq, size = ref.frequencies(hd, 500000.0, "parts", 4.0, 64)
    c = P.PagedCache(layers, heads[0], heads[1], hd, batch, 200, 160, n_blocks=40 * 16 // block, block_size=block, rope=rope, max_new=4)
    book = Book(batch, layers)
    length = [-1] * batch
    # prompts (one slot stays empty), a chunk for some, then drafts of which some tokens are rejected, an end and a newcomer
    steps = [("prompt", [0, 0, -1, 0, 0], [37, 1, 0, 64, 20]), ("chunk", [37, 1, -1, 64, 20], [50, 0, 0, 17, 1]), ("attend", [87, 1, -1, 81, 21], [4, 1, 0, 4, 3]),
             ("attend", [89, 2, -1, 85, 21], [4, 4, 0, 1, 4]), ("prompt", [-1, -1, 0, -1, -1], [0, 0, 23, 0, 0]), ("attend", [0, 0, 23, 0, 0], [1, 2, 4, 0, 1])]
    for n, (how, cached, new) in enumerate(steps):
        if how == "prompt":                                            # these slots begin anew
            for b, p in enumerate(cached):
                if p <= 0:
                    length[b] = p
        rows = sum(new) + n % 3
        c.begin(i32(cached), i32(new), rows)
        for layer in range(layers):
            q, k, v = step_inputs(rng, rows, *heads, hd, dtype)
            q0, k0 = q.clone(), k.clone()
            total = sum(p + m for p, m in zip(cached, new) if p >= 0)
            out = run_step(c, layer, q, k, v, how, total + 3)
            torch.cuda.synchronize()
            check_step(book, layer, cached, new, q0, k0, q, k, v, out, freq, size, dtype, how)
        want = [p + m if p >= 0 else -1 for p, m in zip(cached, new)]
        assert host(c.seq_len).astype(int).tolist() == want
        used = {int(x) for b in range(batch) for x in host(c.table)[b, :int(host(c.owned)[b])]}
        free = {int(x) for x in host(c.free_ids)[:int(host(c.free_count)[0])]}
        assert not used & free and len(used) + len(free) == c.n_blocks and len(used) == int(host(c.owned).sum())


def test_serving_in_a_graph(P):
    """A decode step captured once and replayed, with other eager work between: lengths and rows change, the books go on in place."""
    rng = np.random.default_rng(3)
    batch, hd, heads = 6, 64, (4, 2)
    c = P.PagedCache(1, *heads, hd, batch, 1500, 16, n_blocks=150, block_size=16, max_new=2)
    freq, size = ref.frequencies(hd, 10000.0)
    book = Book(batch, 1)
    cached = [0, 0, 0, 0, 0, 0]
    new = [900, 5, 16, 33, 1, 64]
    big = P.PagedCache(1, *heads, hd, batch, 1500, 1019, n_blocks=150, block_size=16, max_new=2)
    big.pools, big.descs, big.table, big.owned, big.free_ids, big.free_count = c.pools, c.descs, c.table, c.owned, c.free_ids, c.free_count
    big.begin(i32(cached), i32(new), 1019)
    q, k, v = step_inputs(rng, 1019, *heads, hd, "bf16")
    q0, k0 = q.clone(), k.clone()
    out = run_step(big, 0, q, k, v, "attend")
    torch.cuda.synchronize()
    at = 0
    for b, n in enumerate(new):
        book.add(0, b, 0, host(k)[at:at + n], host(v)[at:at + n])
        at += n
    rows = 12
    t_cached, t_new = i32(new), i32([1] * batch)
    q, k, v = step_inputs(rng, rows, *heads, hd, "bf16")
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            c.begin(t_cached, t_new, rows)
            c.rotate(q, k)
            c.append(0, k, v)
            c.attend(0, q, out=out)
    cached = list(new)
    for n in range(6):
        new = [int(x) for x in rng.integers(0, 3, batch)]
        if n == 3:
            cached[1], new[1] = -1, 0                                  # finished
        if n == 4:
            cached[1] = 0                                              # and another in its place
        t_cached.copy_(i32(cached))
        t_new.copy_(i32(new))
        for t in (q, k, v):
            t.copy_(randn(rng, tuple(t.shape), "bf16"))
        q0, k0 = q.clone(), k.clone()
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        check_step(book, 0, cached, new, q0, k0, q, k, v, out, freq, size, "bf16", "attend")
        assert np.all(host(out)[sum(new):] == 7) and torch.equal(q[sum(new):], q0[sum(new):])
        extra = torch.randn(1 << 20, device=DEV).sum().item()          # the program's own work between replays
        assert math.isfinite(extra)
        cached = [p + m if p >= 0 else p for p, m in zip(cached, new)]
        cached = [p - 1 if p > 0 and n % 2 and m == 2 else p for p, m in zip(cached, new)]     # a rejected token


def test_two_caches_on_two_streams(P):
    """Two batches in flight at once, each with its own cache, workspace and stream, give what each gives alone."""
    hd, heads, batch = 128, (8, 2), 4
    results = []
    for together in (False, True):
        torch.manual_seed(1)
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        caches = [P.PagedCache(1, *heads, hd, batch, 3000, 3000, n_blocks=260, block_size=64, max_new=1) for _ in range(2)]
        data = [[torch.randn(2400, n, hd, device=DEV).bfloat16() for n in (heads[0], heads[1], heads[1])] for _ in range(2)]
        lens = [([0] * 4, [600] * 4), ([0] * 4, [1, 2000, 399, 0])]
        one = i32([1] * 4)
        outs = [[], []]
        torch.cuda.synchronize()
        t_lens = [(i32(a), i32(b), i32(np.add(a, b))) for a, b in lens]
        torch.cuda.synchronize()
        for n in range(2):
            with torch.cuda.stream(streams[n]):
                c, (q, k, v) = caches[n], data[n]
                c.begin(t_lens[n][0], t_lens[n][1], 2400)
                outs[n].append(run_step(c, 0, q, k, v, "prompt"))
                c.begin(t_lens[n][2], one, 4)
                q, k, v = q[:4].clone(), k[:4].clone(), v[:4].clone()
                outs[n].append(run_step(c, 0, q, k, v, "attend"))
                if not together:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        results.append([t for pair in outs for t in pair])
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_what_does_not_fit_is_refused_or_left_out(P):
    c = P.PagedCache(1, 4, 2, 64, 2, 64, 8, n_blocks=3, block_size=16)
    with pytest.raises(ValueError):
        c.begin(i32([0, 0]), i32([4, 5]), 9)
    with pytest.raises(ValueError):
        P.PagedCache(1, 4, 2, 96, 2, 64, 8, n_blocks=3, block_size=16)
    with pytest.raises(ValueError):
        P.PagedCache(1, 5, 2, 64, 2, 64, 8, n_blocks=3, block_size=16)
    c.begin(i32([30, 30]), i32([4, 4]), 8)                             # three blocks each, three in all
    torch.cuda.synchronize()
    assert host(c.seq_len).tolist() == [34, -1] and host(c.slot)[4:].tolist() == [-1] * 4
    q = torch.randn(8, 4, 64, device=DEV).bfloat16()
    with pytest.raises(ValueError):
        c.attend(0, q[:7])
    with pytest.raises(ValueError):
        c.append(0, q, q)
    k, v = q[:, :2].contiguous(), q[:, 2:].contiguous()
    c.append(0, k, v)
    out = c.attend(0, q)
    torch.cuda.synchronize()
    assert np.all(host(out)[4:] == 0)
    with pytest.raises(RuntimeError):
        c.attend(0, torch.randn(8, 4, 64, device=DEV))                 # fp32 queries
