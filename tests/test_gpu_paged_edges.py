"""The operators on paged requests where their parts meet: rows and pieces of a context that hold nothing but NaN, lengths between
max_len and the end of the last block, requests that the plan left out, steps without rows, weights far below the largest.
Tolerances are those of test_gpu_paged.py unless said otherwise."""
import math

import numpy as np
import pytest

import paged_reference as ref
from test_gpu_paged import (DEV, DTYPES, Cache, attend, check_attend, check_attend_rows, check_prompt, host, i32, lse_tolerance, ok, prompt, randn,
                            stream, tolerance)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(scope="module")
def P():
    import paper_2603_17573_amd as P
    return P


# ---- attention over the cache: nothing but NaN --------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("total,head_dim", [(1, 64), (33, 128), (129, 64), (1537, 128), (1537, 64)])
def test_a_key_that_is_nan_alone_in_its_part(P, dtype, total, head_dim):
    """The last token's key has a group that is not finite and is all that a wave, or a workgroup, has of the context."""
    rng = np.random.default_rng(total)
    c = Cache(P, rng, [total, 40], 1, head_dim, 16)
    k, v = (randn(rng, (total + 40, 1, head_dim), "f32") for _ in range(2))
    k[total - 1, 0, 3] = math.inf
    c.write(P, k, v)
    q = randn(rng, (3, 2, head_dim), dtype)
    cu = [0, 2, 3] if total > 1 else [0, 1, 3]
    for max_q, max_seq in ((2, max(total, 40)), (32, 1 << 16)):
        out, lse = attend(P, c, q, cu, max_q, max_seq, 0.1)
        check_attend(c, q, out, lse, cu, ref.held(host(k)), ref.held(host(v)), 0.1, dtype)
    last = cu[1] - 1
    assert np.isnan(host(out)[last]).all() and np.isnan(host(lse)[last]).all()
    assert np.isfinite(host(out)[[r for r in range(3) if r != last]]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("total,head_dim", [(1, 128), (50, 64), (3000, 64), (3000, 128)])
def test_a_query_that_is_nan(P, dtype, total, head_dim):
    """All scores of a row are NaN, in one workgroup and in several: NaN, not the answer of a row that sees nothing."""
    rng = np.random.default_rng(total)
    c = Cache(P, rng, [total, total], 2, head_dim, 32)
    k, v = (randn(rng, (2 * total, 2, head_dim), "f32") for _ in range(2))
    c.write(P, k, v)
    q = randn(rng, (2, 4, head_dim), dtype)
    q[0, 1, 5] = math.nan
    for max_seq in (total, 1 << 16):
        out, lse = attend(P, c, q, [0, 1, 2], 1, max_seq, 0.1)
        check_attend(c, q, out, lse, [0, 1, 2], ref.held(host(k)), ref.held(host(v)), 0.1, dtype)
    assert np.isnan(host(out)[0, 1]).all() and np.isnan(host(lse)[0, 1]) and np.isfinite(host(out)[0, [0, 2, 3]]).all()


# ---- a cache with its calls in order --------------------------------------------------------------------------------------

def fill(c, rng, layer, rows, heads, kv_heads, hd, dtype):
    """Rows of a step, rotated and appended."""
    q, k, v = randn(rng, (rows, heads, hd), dtype), randn(rng, (rows, kv_heads, hd), dtype), randn(rng, (rows, kv_heads, hd), dtype)
    c.rotate(q, k)
    c.append(layer, k, v)
    return q, k, v


def test_host_lengths_are_refused(P):
    c = P.PagedCache(1, 4, 2, 64, 2, 64, 8, n_blocks=6, block_size=16)
    here, there = i32([3, 5]), torch.tensor([3, 5], dtype=torch.int32)
    for a, b in ((there, there), (there, here), (here, there)):
        with pytest.raises(ValueError, match="expected"):
            c.begin(a, b, 8)
    torch.cuda.synchronize()
    assert int(c.free_count[0]) == 6


def test_log_sums_of_another_kind_are_refused(P):
    """attend(), prompt() and chunk() write lse as float32 [rows, q_heads]: anything else would be written past its end."""
    c = P.PagedCache(1, 4, 2, 64, 2, 64, 8, n_blocks=6, block_size=16)
    c.begin(i32([0, 0]), i32([3, 5]), 8)
    q, k, v = fill(c, np.random.default_rng(1), 0, 8, 4, 2, 64, "bf16")
    for lse in (torch.zeros(8, 4, dtype=torch.float16, device=DEV), torch.zeros(8, 4, dtype=torch.float64, device=DEV), torch.zeros(7, 4, device=DEV),
                torch.zeros(32, device=DEV), torch.zeros(8, 8, device=DEV)[:, ::2], torch.zeros(4, 8, device=DEV).t(), torch.zeros(8, 4)):
        for call in (lambda: c.attend(0, q, lse=lse), lambda: c.prompt(q, k, v, lse=lse), lambda: c.chunk(0, q, 8, lse=lse)):
            with pytest.raises(ValueError, match="lse"):
                call()
    same = [torch.full((8, 4), 7.0, device=DEV) for _ in range(3)]
    c.attend(0, q, lse=same[0]), c.prompt(q, k, v, lse=same[1]), c.chunk(0, q, 8, lse=same[2])
    torch.cuda.synchronize()
    assert all(np.isfinite(host(x)).all() and np.all(host(x) != 7) for x in same)


@pytest.mark.parametrize("length", [200, 201, 255, 256, 257])
def test_lengths_up_to_the_end_of_the_last_block(P, length):
    """max_len 200 in blocks of 64: what begin() takes, attend() and chunk() compute alike; what it does not take is left out."""
    rng = np.random.default_rng(length)
    c = P.PagedCache(1, 2, 1, 64, 2, 200, 300, n_blocks=8, block_size=64)
    c.begin(i32([0, 0]), i32([length, 3]), length + 3)
    q, k, v = fill(c, rng, 0, length + 3, 2, 1, 64, "bf16")
    outs = c.attend(0, q), c.chunk(0, q, length + 3)
    torch.cuda.synchronize()
    fits = length <= 256
    assert host(c.seq_len).tolist() == [length if fits else -1, 3]
    for out, chunk in zip(outs, (False, True)):
        for a, b, there in ((0, length, fits), (length, length + 3, True)):
            if there:
                check_attend_rows(host(q)[a:b], host(out)[a:b], ref.held(host(k)[a:b]), ref.held(host(v)[a:b]), 0.125, "bf16", chunk=chunk)
            else:
                assert np.all(host(out)[a:b] == 0)


# ---- the buffers that chunks are read back into ------------------------------------------------------------------------------

def test_chunk_buffers_do_not_pile_up(P):
    """Totals that grow step by step, and dtypes in turn: at most twice the largest need per dtype stays."""
    rng = np.random.default_rng(3)
    heads, hd = 2, 64
    c = P.PagedCache(1, 2, heads, hd, 1, 4096, 64, n_blocks=64, block_size=64)
    c.begin(i32([0]), i32([64]), 64)
    q, k, v = fill(c, rng, 0, 64, 2, heads, hd, "bf16")
    want = c.chunk(0, q, 64)
    torch.cuda.synchronize()
    before, need = torch.cuda.memory_allocated(), 0
    for total in range(66, 4097, 66):
        for dtype in (torch.bfloat16, torch.float16):
            c.chunk(0, q.to(dtype), total)
        need = 2 * 2 * total * heads * hd * 2                          # two dtypes, keys and values
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() - before <= 2 * need
    assert torch.equal(c.chunk(0, q, 64), want)
    check_attend_rows(host(q), host(c.chunk(0, q, 4096)), ref.held(host(k)), ref.held(host(v)), 0.125, "bf16", chunk=True)


def test_a_captured_chunk_keeps_its_buffers(P):
    """A graph with a chunk in it, larger chunks of other sizes afterwards, and memory taken by others: every replay gives the same."""
    rng = np.random.default_rng(5)
    heads, hd = (4, 2), 64
    c = P.PagedCache(1, *heads, hd, 2, 2048, 64, n_blocks=64, block_size=64)
    c.begin(i32([0, 0]), i32([20, 40]), 60)
    q, k, v = fill(c, rng, 0, 60, *heads, hd, "bf16")
    out = torch.empty_like(q)
    want = c.chunk(0, q, 60).clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            c.chunk(0, q, 60, out=out)
    for n in range(4):
        c.chunk(0, q, 200 * (n + 1))
        other = [torch.full((1 << 14,), 255, dtype=torch.uint8, device=DEV) for _ in range(40)]
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), n
        assert all(bool((x == 255).all()) for x in other)


def test_prompts_that_were_left_out(P):
    """A request that got no blocks has rows in the step: zeros and minus infinity from prompt() as from attend() and chunk(), its
    neighbours as ever, rows of nobody as they were."""
    rng = np.random.default_rng(2)
    for dtype, hd in (("bf16", 128), ("f16", 64)):
        new = [150, 20, 300, 7, 40]
        c = P.PagedCache(1, 4, 2, hd, 5, 320, 520, n_blocks=16, block_size=16)     # 10 + 2 blocks, then 19 of 4, 1, 3
        cached = [0, 0, 0, -1, 0]
        c.begin(i32(cached), i32(new), 520)
        q, k, v = fill(c, rng, 0, 520, 4, 2, hd, dtype)
        out, lse = torch.full_like(q, 7.0), torch.full((520, 4), 7.0, device=DEV)
        c.prompt(q, k, v, out=out, lse=lse)
        torch.cuda.synchronize()
        assert host(c.seq_len).tolist() == [150, 20, -1, -1, -1]
        cu = np.concatenate([[0], np.cumsum(new)])
        for i in range(2):
            rows = slice(cu[i], cu[i + 1])
            check_prompt(q[rows], k[rows], v[rows], out[rows], lse[rows], [0, new[i]], [0, new[i]], hd ** -0.5, True, dtype)
        assert np.all(host(out)[170:517] == 0) and np.all(np.isneginf(host(lse)[170:517]))
        assert np.all(host(out)[517:] == 7) and np.all(host(lse)[517:] == 7)
        alike = c.attend(0, q, out=torch.full_like(q, 7.0))
        assert np.all(host(alike)[170:517] == 0) and np.all(host(alike)[517:] == 7)


def test_steps_without_rows(P):
    """A step in which requests only end: every call of it is taken and gives nothing."""
    c = P.PagedCache(1, 4, 2, 64, 3, 64, 8, n_blocks=6, block_size=16)
    c.begin(i32([0, 0, -1]), i32([3, 5, 0]), 8)
    c.begin(i32([-1, -1, -1]), i32([0, 0, 0]), 0)
    q, k, v = (torch.empty(0, n, 64, dtype=torch.bfloat16, device=DEV) for n in (4, 2, 2))
    c.rotate(q, k)
    c.append(0, k, v)
    for out in (c.attend(0, q), c.prompt(q, k, v), c.chunk(0, q, 0)):
        assert tuple(out.shape) == (0, 4, 64)
    torch.cuda.synchronize()
    assert int(c.free_count[0]) == 6


def test_no_keys_at_all(P):
    """Queries over no key rows whose tensors have no memory: zeros and minus infinity.  Reading back no rows: nothing."""
    for dtype in ("bf16", "f16"):
        q = torch.ones(5, 2, 128, dtype=DTYPES[dtype], device=DEV)
        k = torch.empty(0, 1, 128, dtype=DTYPES[dtype], device=DEV)
        assert k.data_ptr() == 0
        for causal in (False, True):
            out, lse = prompt(P, q, k, k, [0, 2, 5], [0, 0, 0], 0.1, causal)
            assert np.all(host(out) == 0) and np.all(np.isneginf(host(lse)))
    c = Cache(P, np.random.default_rng(1), [0, 0], 1, 64, 16)
    k, _ = c.read(P)
    assert k.shape[0] == 0


def test_before_the_first_step(P):
    """Without a begin() there are no rows."""
    c = P.PagedCache(1, 4, 2, 64, 3, 64, 8, n_blocks=6, block_size=16)
    q = torch.empty(0, 4, 64, dtype=torch.bfloat16, device=DEV)
    assert c.attend(0, q).shape[0] == 0 and c.chunk(0, q, 0).shape[0] == 0


def test_a_refused_step_leaves_the_last_one(P):
    """begin() with lengths that it refuses: the calls go on with the step before."""
    rng = np.random.default_rng(6)
    c = P.PagedCache(1, 4, 2, 64, 2, 64, 16, n_blocks=6, block_size=16)
    c.begin(i32([0, 0]), i32([3, 5]), 8)
    q, k, v = fill(c, rng, 0, 8, 4, 2, 64, "bf16")
    want = c.attend(0, q)
    for bad in (i32([0, 0, 0]), i32([[0, 0]]), i32([0, 0]).long(), torch.zeros(2, dtype=torch.int32)):
        with pytest.raises(ValueError):
            c.begin(i32([3, 5]), bad, 12)
    assert torch.equal(c.attend(0, q), want) and c.rows == 8


def test_a_device_without_a_number(P):
    """"cuda" is the current device."""
    rng = np.random.default_rng(1)
    c = P.PagedCache(1, 4, 2, 64, 1, 64, 8, n_blocks=6, block_size=16, device="cuda")
    c.begin(i32([0]), i32([5]), 5)
    q, k, v = fill(c, rng, 0, 5, 4, 2, 64, "bf16")
    out = c.attend(0, q)
    torch.cuda.synchronize()
    check_attend_rows(host(q), host(out), ref.held(host(k)), ref.held(host(v)), 0.125, "bf16")


# ---- prompts: weights far below the largest ------------------------------------------------------------------------------------

@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_many_small_weights_beside_a_large_one(P, dtype, head_dim):
    """One key takes nearly all of the weight and has values of zero, 65536 others have exp(-17) = 2^-24.5 of its weight each and
    values of one: the result is their share, 2^-8.5.  A weight is rounded to the rows' dtype relative to itself down to 2^-25 of the
    largest (fp16 numbers are normal from 2^-14 on and weights are held as 2^11 of their ratio), which leaves the usual tolerance without
    an absolute term; the sum over so many keys adds (t + 64) 2^-24 of it."""
    n = 1 << 16
    q = torch.zeros(3, 2, head_dim, dtype=DTYPES[dtype], device=DEV)
    q[..., 0] = 1
    k = torch.zeros(n + 1, 1, head_dim, dtype=DTYPES[dtype], device=DEV)
    v = torch.ones(n + 1, 1, head_dim, dtype=DTYPES[dtype], device=DEV)
    for at in (0, 700, n):                                             # met first, in the middle, last
        k.zero_()
        v.fill_(1)
        k[at, 0, 0], v[at] = 17.0, 0
        out, lse = prompt(P, q, k, v, [0, 3], [0, n + 1], 1.0, False)
        small = n * math.exp(-17.0)
        want = np.full((3, 2, head_dim), small / (1 + small))
        size = np.full((3, 2), 17.0)
        tol = tolerance(dtype, ref.half_step(dtype), 0.0, head_dim, n + 1, want, want, 0.0, size)
        assert np.all(np.abs(host(out) - want) <= tol), (at, host(out).min(), host(out).max(), want.max(), tol.max())
        assert np.all(np.abs(host(lse) - 17.0 - math.log1p(small)) <= lse_tolerance(head_dim, n + 1, 17.0, size))


@pytest.mark.parametrize("head_dim,causal", [(64, True), (128, False)])
def test_fp16_weights_at_their_largest(P, head_dim, causal):
    """Scores that creep up by less than what moves the maximum, and large values: nothing overflows."""
    rng = np.random.default_rng(9)
    n = 900
    q = torch.zeros(n, 1, head_dim, dtype=torch.float16, device=DEV)
    q[..., 0] = 1
    v = (randn(rng, (n, 1, head_dim), "f32") * 9000).clamp(-65000, 65000).to(torch.float16)
    for step in (0.69 / 64, 1.3 / 64, 5.5 / 64, -0.02):
        k = torch.zeros(n, 1, head_dim, dtype=torch.float16, device=DEV)
        k[:, 0, 0] = torch.arange(n, device=DEV) * step
        out, lse = prompt(P, q, k, v, [0, n], [0, n], 1.0, causal)
        check_prompt(q, k, v, out, lse, [0, n], [0, n], 1.0, causal, "f16")


def test_one_row_or_head_has_any_stride(P):
    """What lies on nothing else is taken whatever its strides say; so are broadcast inputs."""
    rng = np.random.default_rng(4)
    q = randn(rng, (1, 4, 64), "bf16")
    k = randn(rng, (1, 1, 64), "bf16")
    one = torch.full((1, 4, 64), 7.0, dtype=torch.bfloat16, device=DEV).as_strided((1, 4, 64), (8, 64, 1))
    out, lse = prompt(P, q, k, k, [0, 1], [0, 1], 0.125, True, out=one)
    check_prompt(q, k, k, out, lse, [0, 1], [0, 1], 0.125, True, "bf16")
    q = randn(rng, (5, 1, 64), "bf16")
    k = randn(rng, (1, 1, 64), "bf16").expand(40, 1, 64)
    one = torch.full((5, 1, 64), 7.0, dtype=torch.bfloat16, device=DEV).as_strided((5, 1, 64), (64, 8, 1))
    out, lse = prompt(P, q, k, k, [0, 5], [0, 40], 0.125, True, out=one)
    check_prompt(q, k, k, out, lse, [0, 5], [0, 40], 0.125, True, "bf16")
    x = randn(rng, (1, 2, 64), "f32").expand(6, 2, 64)
    turns, size = P.rope_table(P.make_rope_desc(64), DEV)
    y, pos = torch.empty(6, 2, 64, device=DEV), i32(range(6))
    ok(P, P.heisd_rope(turns.data_ptr(), size, 64, 0, 0, pos.data_ptr(), 6, 64, P.head_rows(x), P.head_rows(y), None, None, stream()))
    torch.cuda.synchronize()
    freq, _ = ref.frequencies(64, 10000.0)
    assert np.abs(host(y) - ref.rope(host(x), np.arange(6), freq, 1.0, "half", False)).max() <= 2.0 ** -20 * float(x.abs().max())
    with pytest.raises(RuntimeError, match="on each other"):
        c = P.PagedCache(1, 2, 2, 64, 1, 64, 8, n_blocks=6, block_size=16)
        c.begin(i32([0]), i32([6]), 6)
        c.rotate(x, y)


def test_log_sums_made_for_larger_steps(P):
    """An lse of more rows than the step has: the first ones are written, the others left."""
    c = P.PagedCache(1, 4, 2, 64, 2, 64, 16, n_blocks=6, block_size=16)
    c.begin(i32([0, 0]), i32([3, 5]), 8)
    q, k, v = fill(c, np.random.default_rng(1), 0, 8, 4, 2, 64, "bf16")
    for call in (lambda x: c.attend(0, q, lse=x), lambda x: c.prompt(q, k, v, lse=x), lambda x: c.chunk(0, q, 8, lse=x)):
        exact, more = torch.full((8, 4), 7.0, device=DEV), torch.full((16, 4), 7.0, device=DEV)
        call(exact), call(more)
        torch.cuda.synchronize()
        assert torch.equal(more[:8], exact) and bool((more[8:] == 7).all()) and bool((exact != 7).all())
