"""Block tables, rotary positions, the cache in 4 bits with its attention, and attention of packed prompts through the C ABI,
against the plain definitions of paged_reference.py.

Tolerances.  A rounding to a dtype is off by at most half a step, u = eps / 2 of the value (bf16 2^-8, fp16 2^-11, fp32 2^-24).
Whole numbers and what a 4-bit cache holds are exact.  Rotations: u of the result, and in fp32 two products, a sum (2^-24 each)
and sine and cosine to 2^-22.  Attention: a score is a sum of head_dim products in fp32, each addition off by 2^-24 of what has been summed, so
off by at most S = (head_dim + 8) 2^-24 * scale * sum |q_i k_i|, which makes a probability relatively off by exp(2 S) - 1 (its own
score and the normalising sum); the probability's own rounding P adds 2^-16 (a bf16 and a remainder of a bf16: over the cache) or
the rows' own u (in prompts), where fp16 probabilities below 2^-14 are off by 2^-25 at most; the sums of the output over t tokens
add (t + 64) 2^-24.  All of these multiply the weighted mean of |v|; the result is rounded once."""
import math

import numpy as np
import pytest

import paged_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(scope="module")
def P():
    import paper_2603_17573_amd as P
    return P


def ok(P, rc):
    assert rc == 0, P.heisd_last_error(None)


def i32(values):
    return torch.tensor(np.asarray(values), dtype=torch.int32, device=DEV)


def host(t):
    return t.detach().double().cpu().numpy()


def randn(rng, shape, dtype, spread=True):
    x = rng.standard_normal(shape)
    if spread:
        x = x * np.exp(0.5 * rng.standard_normal(shape[-2:]))
    return torch.tensor(x, device=DEV).to(DTYPES[dtype])


def stream():
    return torch.cuda.current_stream().cuda_stream


# ---- block tables ---------------------------------------------------------------------------------------------------

def books(rng, batch, block, max_blocks, cached_most, new_most, spare, finished=0.2, pad=0):
    cached = [int(rng.integers(0, cached_most + 1)) for _ in range(batch)]
    new = [int(rng.integers(0, new_most + 1)) for _ in range(batch)]
    owned = [min(max_blocks, -(-c // block) + int(rng.integers(0, 2))) for c in cached]      # some own a block more than they use
    for i in range(batch):
        if rng.random() < finished:
            cached[i], new[i] = -1, int(rng.integers(0, 2))
    n_blocks = sum(owned) + max(spare, 1)
    ids = rng.permutation(n_blocks)
    table = np.full((batch, max_blocks), -1, np.int64)
    at = 0
    for i, n in enumerate(owned):
        table[i, :n] = ids[at:at + n]
        at += n
    free_ids = np.full(n_blocks, -1, np.int64)
    free_ids[:n_blocks - at] = ids[at:]
    return dict(cached=cached, new=new, owned=owned, table=table, free_ids=free_ids, free_count=min(spare, n_blocks - at), block=block,
                n_blocks=n_blocks, rows=sum(max(n, 0) for n in new) + pad)


def run_plan(P, s, in_place=False, cu_seq=True):
    b, t = len(s["cached"]), {}
    for k in ("cached", "new", "owned", "table", "free_ids"):
        t[k] = i32(s[k])
    t["free_count"] = i32([s["free_count"]])
    out = {"owned": t["owned"] if in_place else torch.full((b,), -7, dtype=torch.int32, device=DEV),
           "free_count": t["free_count"] if in_place else i32([-7]), "seq_len": i32([-7] * b), "cu_rows": i32([-7] * (b + 1)),
           "slot": i32([-7] * s["rows"]), "position": i32([-7] * s["rows"]), "table": t["table"], "free_ids": t["free_ids"]}
    if cu_seq:
        out["cu_seq"] = i32([-7] * (b + 1))
    d = P.make_plan_desc(s["block"], s["n_blocks"], t["cached"], t["new"], t["owned"], out["owned"], t["table"], t["free_ids"],
                         t["free_count"], out["free_count"], out["seq_len"], out["cu_rows"], out["slot"], out["position"],
                         out.get("cu_seq"))
    ok(P, P.heisd_paged_plan(d, stream()))
    torch.cuda.synchronize()
    return out, (d, t)


def check_plan(s, out):
    want = ref.plan(s["cached"], s["new"], s["owned"], s["table"], s["free_ids"], s["free_count"], s["rows"], s["block"], s["n_blocks"])
    for k in out:
        assert np.array_equal(np.atleast_1d(host(out[k]).astype(np.int64)), np.atleast_1d(np.asarray(want[k]))), k


@pytest.mark.parametrize("batch,block,cached,new,spare,pad", [
    (1, 16, 0, 1, 4, 0), (1, 16, 276, 7, 4, 0), (1, 64, 0, 5000, 90, 0), (7, 16, 40, 40, 100, 5), (64, 32, 600, 3, 70, 0),
    (1023, 16, 50, 4, 2000, 1), (1025, 16, 60, 9, 3000, 0), (2600, 1, 9, 3, 9000, 130), (512, 64, 4000, 200, 3000, 3), (3, 48, 100, 9, 12, 2)])
@pytest.mark.parametrize("in_place", [False, True])
def test_plan(P, batch, block, cached, new, spare, pad, in_place):
    rng = np.random.default_rng(batch * 1000 + block + cached)
    s = books(rng, batch, block, -(-(cached + new) // block) + 1, cached, new, spare, pad=pad)
    check_plan(s, run_plan(P, s, in_place, cu_seq=not in_place)[0])


def test_plan_leaves_out_what_does_not_fit(P):
    """Too few blocks (and nobody after the first refusal is served with new ones), too long for the table, negative new
    lengths, more rows than there are."""
    rng = np.random.default_rng(5)
    for spare in (0, 1, 5, 9):
        check_plan(*(lambda s: (s, run_plan(P, s)[0]))(books(rng, 40, 16, 8, 60, 60, spare, finished=0.1)))
    s = books(rng, 12, 16, 8, 60, 60, 500, finished=0.1)
    s["cached"][3], s["new"][3] = 100, 29                             # 129 tokens, the table holds 128
    s["cached"][4], s["new"][4] = 100, 28
    s["new"][6] = -5
    s["cached"][7], s["new"][7] = 2 ** 31 - 1, 2                      # the sum passes 32 bits
    s["rows"] = sum(max(n, 0) for n in s["new"])
    check_plan(s, run_plan(P, s)[0])
    s["rows"] -= 10                                                   # the last requests' rows are not there
    check_plan(s, run_plan(P, s)[0])
    s["new"][2] = 2 ** 31 - 1                                         # nor anything from here on, and the sums pass 32 bits
    s["new"][9] = 2 ** 31 - 1
    check_plan(s, run_plan(P, s)[0])


def test_plan_with_table_entries_out_of_range(P):
    s = dict(cached=[20, 20], new=[3, 3], owned=[2, 2], table=np.array([[0, 9, -1], [3, -5, -1]]), free_ids=np.array([1, 2, -1, -1]),
             free_count=2, block=16, n_blocks=4, rows=6)
    check_plan(s, run_plan(P, s)[0])


def test_plan_twice_gives_the_same(P):
    """The small inputs are not changed (separate outputs): the same call again does the same work and leaves the same state."""
    s = books(np.random.default_rng(8), 300, 16, 12, 90, 70, 900)
    out, (d, keep) = run_plan(P, s)
    first = {k: v.clone() for k, v in out.items()}
    ok(P, P.heisd_paged_plan(d, stream()))
    torch.cuda.synchronize()
    for k in out:
        assert torch.equal(out[k], first[k]), k


# ---- rotary positions -------------------------------------------------------------------------------------------------

def run_rope(P, q, k, position, rotary, layout="half", inverse=False, in_place=False, **desc):
    turns, size = P.rope_table(P.make_rope_desc(rotary, **desc), DEV)
    qo, ko = (q, k) if in_place else (torch.full_like(q, 7.0), torch.full_like(k, 7.0) if k is not None else None)
    hr = lambda t: P.head_rows(t) if t is not None else None  # noqa: E731
    ok(P, P.heisd_rope(turns.data_ptr(), size, rotary, P.ROPE_LAYOUT[layout], int(inverse), position.data_ptr(), q.shape[0], q.shape[2],
                       hr(q), hr(qo), hr(k), hr(ko), stream()))
    torch.cuda.synchronize()
    return qo, ko


def check_rope(x, y, position, freq, size, layout, inverse, dtype, before=7.0):
    x, y, pos = host(x), host(y), host(position)
    want = ref.rope(x, pos, freq, size, layout, inverse)
    n = 2 * len(freq)
    pair = np.abs(x[..., :n // 2]) + np.abs(x[..., n // 2:n]) if layout == "half" else np.abs(x[..., 0:n:2]) + np.abs(x[..., 1:n:2])
    pair = np.concatenate([pair, pair], -1) if layout == "half" else np.repeat(pair, 2, -1)
    tol = ref.half_step(dtype) * np.abs(want) + 2.0 ** -25
    tol[..., :n] += (2 * 2.0 ** -24 + 2.0 ** -22) * size * pair
    tol[..., n:] = 0
    live = pos >= 0
    assert np.all(np.abs(y - want)[live] <= tol[live])
    if before is not None:
        assert np.all(y[~live] == before)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype,rows,heads,head_dim,rotary", [
    ("bf16", 1, (1, 1), 64, 64), ("bf16", 7, (32, 32), 128, 128), ("bf16", 2500, (8, 2), 128, 64), ("f16", 33, (5, 1), 128, 96),
    ("f32", 300, (4, 4), 64, 32), ("f32", 5, (3, 2), 256, 256), ("bf16", 9, (2, 1), 80, 20), ("f16", 3, (2, 2), 7, 6), ("f32", 4100, (2, 1), 2, 2)])
def test_rope(P, layout, dtype, rows, heads, head_dim, rotary):
    rng = np.random.default_rng(rows + head_dim)
    q, k = (randn(rng, (rows, h, head_dim), dtype) for h in heads)
    position = i32(rng.integers(-1, 4096, rows))
    freq, size = ref.frequencies(rotary, 10000.0)
    for inverse in (False, True):
        qo, ko = run_rope(P, q, k, position, rotary, layout, inverse)
        check_rope(q, qo, position, freq, size, layout, inverse, dtype)
        check_rope(k, ko, position, freq, size, layout, inverse, dtype)


@pytest.mark.parametrize("scaling", ["none", "linear", "base", "parts", "bands"])
def test_rope_scalings_at_far_positions(P, scaling):
    rng = np.random.default_rng(3)
    more = dict(factor=8.0, original_len=8192) if scaling != "none" else {}
    q, k = randn(rng, (64, 3, 128), "f32"), randn(rng, (64, 1, 128), "f32")
    position = i32(np.concatenate([rng.integers(0, 2 ** 31 - 1, 60), [0, 1, 131071, 2 ** 31 - 1]]))
    freq, size = ref.frequencies(128, 500000.0, scaling, more.get("factor", 1.0), more.get("original_len", 0))
    qo, ko = run_rope(P, q, k, position, 128, base=500000.0, scaling=scaling, **more)
    # 64-bit angles of positions up to 2^31 are themselves off by 2^31 * 2^-53 of a radian, in the reference too
    check_rope(q, qo, position, freq, size, "half", False, "f32")
    check_rope(k, ko, position, freq, size, "half", False, "f32")


def test_rope_layouts_in_place_without_keys(P):
    """Head-major rows, rows of a wider matrix, unaligned rows, in place, no keys, negative positions untouched."""
    rng = np.random.default_rng(4)
    position = i32([5, -1, 0, 700, -3, 12])
    freq, size = ref.frequencies(64, 10000.0)
    wide = randn(rng, (6, 11, 64), "bf16")
    for make in (lambda: wide.transpose(0, 1).contiguous().transpose(0, 1), lambda: wide[:, 2:7], lambda: wide[:, ::2],
                 lambda: randn(rng, (6, 5, 65), "bf16")[..., 1:], lambda: randn(rng, (6, 5, 72), "bf16")[..., 4:68]):
        for in_place in (False, True):
            q = make()
            x = q.clone()
            whole = q._base.clone() if q._base is not None else None
            qo, _ = run_rope(P, q, None, position, 64, in_place=in_place)
            want_rest = host(x)[[1, 4]] if in_place else 7.0
            check_rope(x, qo, position, freq, size, "half", False, "bf16", before=None)
            assert np.all(host(qo)[[1, 4]] == want_rest)
            if in_place and whole is not None:                         # nothing beside the view
                q.copy_(x)
                assert torch.equal(q._base, whole)


def test_rope_gradient_is_the_inverse_call(P):
    """<g, R x> = <R^T g, x> for the library's own R and R^T, and against differences of R."""
    rng = np.random.default_rng(6)
    for layout, scaling in (("half", "parts"), ("interleaved", "bands")):
        x, g = randn(rng, (40, 2, 64), "f32"), randn(rng, (40, 2, 64), "f32")
        position = i32(rng.integers(0, 9000, 40))
        more = dict(rotary=48, layout=layout, scaling=scaling, factor=4.0, original_len=512)
        y, _ = run_rope(P, x, None, position, **more)
        gx, _ = run_rope(P, g, None, position, inverse=True, **more)
        left, right, terms = (host(g) * host(y)).sum(), (host(gx) * host(x)).sum(), np.abs(host(g) * host(y)).sum()
        # every product is off by (2 + 4) 2^-24 of the pair's magnitudes (above); their sum is at most 2 sqrt(2) times the terms' here
        assert abs(left - right) <= 2 ** -20 * max(terms, np.abs(host(gx) * host(x)).sum()) * 3
        d = randn(rng, (40, 2, 64), "f32")
        y2, _ = run_rope(P, x + d, None, position, **more)
        # a linear map: the difference quotient is exact but for rounding
        diff = (host(g) * (host(y2) - host(y))).sum()
        assert abs(diff - (host(gx) * (host(x + d) - host(x))).sum()) <= 2 ** -20 * 6 * np.abs(host(g) * np.abs(host(y2)) + np.abs(host(y))).sum()


# ---- the cache ------------------------------------------------------------------------------------------------------------

class Cache:
    """A pool with tables of shuffled blocks for requests of `total` tokens, full of rubbish (255 everywhere) to begin with."""

    def __init__(self, P, rng, total, kv_heads, head_dim, block, spare=2):
        need = [-(-n // block) for n in total]
        self.n_blocks, self.block, self.kv_heads, self.head_dim, self.total = sum(need) + spare, block, kv_heads, head_dim, total
        self.pool = torch.full((P.heisd_kv4_pool_bytes(self.n_blocks, block, kv_heads, head_dim),), 255, dtype=torch.uint8, device=DEV)
        self.desc = P.make_kv4_desc(self.pool, block, kv_heads, head_dim)
        ids = rng.permutation(self.n_blocks)
        self.table = np.full((len(total), max(1, max(need)) + 1), -1, np.int64)
        at = 0
        for i, n in enumerate(need):
            self.table[i, :n] = ids[at:at + n]
            at += n
        self.t_table, self.t_seq = i32(self.table), i32(total)
        self.cu_seq = np.concatenate([[0], np.cumsum(np.maximum(total, 0))])

    def slots(self):
        """Of all tokens of all requests, packed."""
        return np.concatenate([self.table[i, np.arange(n) // self.block] * self.block + np.arange(n) % self.block
                               for i, n in enumerate(self.total)] + [np.zeros(0, np.int64)])

    def batch(self, P, cu_rows, rows):
        self.t_cu = i32(cu_rows)
        return P.make_paged_batch(self.t_table, self.t_seq, self.t_cu, rows)

    def write(self, P, k, v, slots=None):
        t = i32(self.slots() if slots is None else slots)
        ok(P, P.heisd_kv4_append(self.desc, P.head_rows(k), P.head_rows(v), t.data_ptr(), k.shape[0], stream()))
        torch.cuda.synchronize()

    def read(self, P, dtype="f32", rows=None, extra=0, cu_seq=None):
        rows = int(self.cu_seq[-1]) + extra if rows is None else rows
        k, v = (torch.full((rows, self.kv_heads, self.head_dim), 7.0, dtype=DTYPES[dtype], device=DEV) for _ in range(2))
        cu = i32(self.cu_seq if cu_seq is None else cu_seq)
        ok(P, P.heisd_kv4_gather(self.desc, self.batch(P, [0] * (len(self.total) + 1), 0), cu.data_ptr(), rows, P.head_rows(k),
                                 P.head_rows(v), stream()))
        torch.cuda.synchronize()
        return k, v


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("total,kv_heads,head_dim,block", [([1], 1, 64, 16), ([33, 0, 5], 3, 128, 16), ([17, 64, 1], 2, 64, 64), ([70], 8, 128, 32),
                                                           ([3] * 40, 1, 128, 128)])
def test_cache_holds_what_the_format_says(P, dtype, total, kv_heads, head_dim, block):
    rng = np.random.default_rng(len(total) + head_dim)
    c = Cache(P, rng, total, kv_heads, head_dim, block)
    n = sum(total)
    x = rng.standard_normal((2, n, kv_heads, head_dim)) * np.exp(3 * rng.standard_normal((2, n, kv_heads, 1)))
    x[0, 0, 0, :32] = 0                                                # a group of zeros
    x[1, 0, 0, :32] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6] * 4     # ties, and the largest value in place
    x[0, -1, -1, 32:64] = -np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6] * 4) * 2.0 ** -9
    x[1, -1, -1, :32] = 0
    x[1, -1, -1, 0] = 6.0 + 2.0 ** -4                                  # just above 6: the next power of two
    x[1, -1, -1, 1] = 1e-4
    k, v = (torch.tensor(y, device=DEV).to(DTYPES[dtype]) for y in x)
    c.write(P, k, v)
    want_k, want_v = ref.held(host(k)), ref.held(host(v))
    gk, gv = c.read(P, extra=2)
    assert np.array_equal(host(gk)[:n], want_k) and np.array_equal(host(gv)[:n], want_v)
    assert np.all(host(gk)[n:] == 7) and np.all(host(gv)[n:] == 7)
    for out in ("bf16", "f16"):
        gk, gv = c.read(P, out)
        assert torch.equal(gk, torch.tensor(want_k, device=DEV).to(DTYPES[out])) and torch.equal(gv, torch.tensor(want_v, device=DEV).to(DTYPES[out]))


def test_cache_extremes(P):
    """Subnormal, largest and non-finite fp32 values; a group that is not finite reads as NaN, its neighbours do not."""
    rng = np.random.default_rng(0)
    c = Cache(P, rng, [4], 1, 64, 16)
    x = rng.standard_normal((4, 1, 64)).astype(np.float32)
    x[0, 0, :32] *= np.float32(2.0 ** -140)
    x[0, 0, 32:] *= np.float32(2.0 ** -127)
    x[1, 0, :32] = np.float32(3.4e38) * np.sign(x[1, 0, :32])
    x[2, 0, 3] = np.inf
    x[3, 0, 40] = np.nan
    t = torch.tensor(x, device=DEV)
    c.write(P, t, t.flip(0).contiguous())
    gk, gv = c.read(P)
    with np.errstate(invalid="ignore", over="ignore"):                 # 3.4e38 is held as 4 * 2^126, which fp32 rounds to infinity
        want_k, want_v = (ref.held(y).astype(np.float32) for y in (x, x[::-1].copy()))
    assert np.array_equal(host(gk), want_k, equal_nan=True) and np.array_equal(host(gv), want_v, equal_nan=True)
    assert np.isnan(host(gk)[2, 0, :32]).all() and np.isfinite(host(gk)[2, 0, 32:]).all()


def test_cache_rows_anywhere(P):
    """Rows of a wider matrix, head-major, unaligned and broadcast rows; negative and too large slots change nothing."""
    rng = np.random.default_rng(9)
    c = Cache(P, rng, [20], 2, 64, 16, spare=1)
    a = randn(rng, (20, 7, 64), "bf16")
    b = randn(rng, (2, 20, 64), "bf16").transpose(0, 1)
    odd = randn(rng, (20, 2, 67), "bf16")[..., 2:66]
    one = randn(rng, (1, 2, 64), "bf16").expand(20, 2, 64)
    for k, v in ((a[:, 1:3], b), (odd, a[:, 4:6]), (one, odd)):
        c.write(P, k, v)
        gk, gv = c.read(P, "f32")
        assert np.array_equal(host(gk), ref.held(host(k))) and np.array_equal(host(gv), ref.held(host(v)))
    before = c.pool.clone()
    size = c.n_blocks * c.block
    c.write(P, a[:, :2], b, slots=[-1, size, 2 ** 31 - 1, -2 ** 31] * 5)
    assert torch.equal(c.pool, before)
    # outputs in another order, and beside them nothing
    big = torch.full((2, 25, 80), 7.0, dtype=torch.bfloat16, device=DEV)
    k_out, v_out = big.transpose(0, 1)[2:22, :, 9:73], torch.empty((20, 2, 64), dtype=torch.bfloat16, device=DEV)
    cu = i32([0, 20])
    ok(P, P.heisd_kv4_gather(c.desc, c.batch(P, [0, 0], 0), cu.data_ptr(), 20, P.head_rows(k_out), P.head_rows(v_out), stream()))
    torch.cuda.synchronize()
    assert torch.equal(k_out.float(), gk) and torch.equal(v_out.float(), gv)
    k_out.fill_(7.0)
    assert bool((big == 7).all())


def test_gather_of_what_is_not_there(P):
    """Missing blocks give zeros; requests without tokens, spans longer than the request and rows of nobody are left alone; spans
    that make no sense touch nothing."""
    rng = np.random.default_rng(2)
    c = Cache(P, rng, [40, 3, 20], 1, 64, 16)
    k, v = randn(rng, (63, 1, 64), "f32"), randn(rng, (63, 1, 64), "f32")
    c.write(P, k, v)
    c.table[0, 1] = c.n_blocks
    c.table[2, 0] = -4
    c.t_table, c.t_seq = i32(c.table), i32([40, -1, 20])
    gk, _ = c.read(P, rows=70, cu_seq=[0, 43, 46, 69])
    want = ref.held(host(k))
    got = host(gk)
    assert np.array_equal(got[:16], want[:16]) and np.all(got[16:32] == 0) and np.array_equal(got[32:40], want[32:40])
    assert np.all(got[40:46] == 7) and np.all(got[46:62] == 0) and np.array_equal(got[62:66], want[59:63]) and np.all(got[66:] == 7)
    gk, _ = c.read(P, rows=10, cu_seq=[5, -3, 90, 12])
    assert np.all(host(gk) == 7)


# ---- attention ---------------------------------------------------------------------------------------------------------------

def tolerance(dtype, p_rounding, tiny, head_dim, tokens, want, mean, flat, size, scale_terms=0.0):
    s = (head_dim + 8) * 2.0 ** -24 * size[..., None] + 2.0 ** -22 * (size[..., None] + 1) + scale_terms
    p = np.expm1(2 * s) + p_rounding + (tokens + 64) * 2.0 ** -24
    return p * mean + tiny * flat + ref.half_step(dtype) * np.abs(want) + 2.0 ** -25


def lse_tolerance(head_dim, tokens, lse, size):
    return 2 * ((head_dim + 8) * 2.0 ** -24 * size + 2.0 ** -22 * (size + 1)) + (tokens + 64) * 2.0 ** -24 + 2.0 ** -22 * np.abs(np.where(np.isfinite(lse), lse, 0))


def attend(P, c, q, cu_rows, max_q, max_seq, scale, want_lse=True, workspace=None, out=None):
    rows = q.shape[0]
    out = torch.full_like(q, 7.0) if out is None else out
    lse = torch.full(q.shape[:2], 7.0, device=DEV) if want_lse else None
    n = P.heisd_kv4_attention_workspace_bytes(c.desc, len(c.total), rows, q.shape[1], max_q, max_seq)
    assert n > 0
    ws = torch.full((n,), 255, dtype=torch.uint8, device=DEV) if workspace is None else workspace
    b = c.batch(P, cu_rows, rows)
    ok(P, P.heisd_kv4_attention(c.desc, b, P.head_rows(q), P.head_rows(out), lse.data_ptr() if want_lse else None, scale, max_q, max_seq,
                                ws.data_ptr(), n, stream()))
    torch.cuda.synchronize()
    return out, lse


def check_attend(c, q, out, lse, cu_rows, k, v, scale, dtype, seq=None, gone=None):
    """k, v: what the cache holds, packed by request [sum(total), kv_heads, head_dim]."""
    seq = c.total if seq is None else seq
    q64, out, lse = host(q), host(out), host(lse)
    p = 2.0 ** -16
    for i, n in enumerate(seq):
        a, b = cu_rows[i], cu_rows[i + 1]
        kk, vv = (x[c.cu_seq[i]:c.cu_seq[i] + max(n, 0)] for x in (k, v))
        keep = np.ones(max(n, 0), bool) if gone is None else ~gone[i][:max(n, 0)]
        for r in range(a, b):
            t = min(max(n - (b - a) + (r - a) + 1, 0), max(n, 0))
            live = keep[:t]
            want, wl, mean, flat, size = ref.attention(q64[r:r + 1], kk[:t][live], vv[:t][live], [int(live.sum())], scale)
            nan = np.isnan(want)
            assert np.array_equal(np.isnan(out[r:r + 1]), nan)
            tol = tolerance(dtype, p, 0.0, q.shape[2], t, want, mean, flat, size)
            assert np.all((np.abs(out[r:r + 1] - want) <= tol)[~nan]), (i, r, np.nanmax(np.abs(out[r] - want)))
            fine = np.isfinite(wl)
            assert np.array_equal(lse[r:r + 1][~fine], wl[~fine], equal_nan=True)
            assert np.all(np.abs(lse[r:r + 1][fine] - wl[fine]) <= lse_tolerance(q.shape[2], t, wl, size)[fine])


def check_attend_rows(q, out, k, v, scale, dtype, chunk=False):
    """The n rows of one request over all that it has cached; chunk: by way of packed rows in the queries' dtype."""
    n, t = q.shape[0], k.shape[0]
    want, _, mean, flat, size = ref.attention(q, k, v, [t - n + i + 1 for i in range(n)], scale)
    p, tiny = (2.0 ** -16, 0.0) if not chunk else (2.0 ** -8, 0.0) if dtype == "bf16" else (2.0 ** -11, 2.0 ** -25)
    over = np.abs(out - want) - tolerance(dtype, p, tiny, q.shape[2], t, want, mean, flat, size)
    assert over.max() <= 0, (chunk, n, t, float(over.max()), np.argwhere(over > 0)[:4].tolist())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("total,new,heads,head_dim,block", [
    ([1], [1], (1, 1), 64, 16), ([1, 2, 15, 16, 17, 31, 33], [1] * 7, (4, 2), 128, 16), ([127, 128, 129, 300], [1, 2, 1, 3], (8, 1), 128, 32),
    ([283], [7], (4, 4), 128, 16), ([40, 7, 100], [7, 7, 7], (4, 1), 64, 64), ([5, 90], [5, 40], (6, 2), 128, 16), ([600, 0, 3], [2, 0, 1], (5, 1), 64, 128),
    ([1500], [1], (32, 8), 128, 16), ([20, 20], [0, 14], (16, 2), 64, 16)])
def test_attention_over_the_cache(P, dtype, total, new, heads, head_dim, block):
    rng = np.random.default_rng(sum(total) + head_dim + heads[0])
    c = Cache(P, rng, total, heads[1], head_dim, block)
    k, v = (randn(rng, (sum(total), heads[1], head_dim), "bf16") for _ in range(2))
    c.write(P, k, v)
    cu = np.concatenate([[0], np.cumsum(new)])
    q = randn(rng, (int(cu[-1]) + 2, heads[0], head_dim), dtype)
    scale = 1 / math.sqrt(head_dim)
    out, lse = attend(P, c, q, cu, max(new), max(total), scale)
    check_attend(c, q, out, lse, cu, ref.held(host(k)), ref.held(host(v)), scale, dtype)
    assert np.all(host(out)[cu[-1]:] == 7) and np.all(host(lse)[cu[-1]:] == 7)
    again, _ = attend(P, c, q, cu, max(new), max(total), scale, want_lse=False)
    assert torch.equal(again, out)
    # other bounds cut the work otherwise; with the larger ones a workgroup takes 32 columns
    for max_q, max_seq in ((1, 4096), (32, 1 << 20)):
        more, lse = attend(P, c, q, cu, max_q, max_seq, scale)
        check_attend(c, q, more, lse, cu, ref.held(host(k)), ref.held(host(v)), scale, dtype)


def test_attention_of_long_contexts(P):
    """Many chunks per request beside short ones; scores that grow along the context, so that the maximum keeps moving."""
    rng = np.random.default_rng(12)
    total = [5000, 1, 4096, 2600]
    c = Cache(P, rng, total, 2, 128, 64)
    k, v = randn(rng, (sum(total), 2, 128), "bf16"), randn(rng, (sum(total), 2, 128), "bf16")
    q = randn(rng, (4, 8, 128), "bf16")
    ramp = torch.linspace(-30, 30, 5000, device=DEV)[:, None, None]
    k[:5000] = (k[:5000].float() * 0.2 + ramp * torch.sign(q[0, ::4].float())[None] / 8).to(k.dtype)
    c.write(P, k, v)
    for max_seq in (5000, 20000):
        out, lse = attend(P, c, q, [0, 1, 2, 3, 4], 1, max_seq, 0.088)
        check_attend(c, q, out, lse, [0, 1, 2, 3, 4], ref.held(host(k)), ref.held(host(v)), 0.088, "bf16")


@pytest.mark.parametrize("batch,heads,head_dim", [(64, (2, 1), 64), (65, (4, 2), 128), (130, (2, 2), 64), (333, (1, 1), 64)])
def test_attention_of_many_requests(P, batch, heads, head_dim):
    """More requests than a wave looks at together; some without rows, some without tokens."""
    rng = np.random.default_rng(batch)
    total = [int(x) for x in rng.integers(0, 300, batch)]
    new = [int(min(x, max(t, 1))) for x, t in zip(rng.integers(0, 3, batch), total)]
    c = Cache(P, rng, total, heads[1], head_dim, 16)
    k, v = (randn(rng, (sum(total), heads[1], head_dim), "bf16") for _ in range(2))
    c.write(P, k, v)
    cu = np.concatenate([[0], np.cumsum(new)])
    q = randn(rng, (int(cu[-1]), heads[0], head_dim), "bf16")
    for max_q in (2, 32):
        out, lse = attend(P, c, q, cu, max_q, 300, 0.1)
        check_attend(c, q, out, lse, cu, ref.held(host(k)), ref.held(host(v)), 0.1, "bf16")


def test_attention_of_long_runs(P):
    """So much work that a workgroup has more than 4096 tokens of one request and head."""
    rng = np.random.default_rng(0)
    total, heads, hd = [8192, 8000, 8191, 4097, 8192, 8100, 8192, 8192], 64, 64
    c = Cache(P, rng, total, heads, hd, 64)
    g = torch.Generator(device=DEV).manual_seed(1)
    k, v = (torch.randn((sum(total), heads, hd), generator=g, device=DEV).bfloat16() for _ in range(2))
    c.write(P, k, v)
    kk, vv = c.read(P)
    q = torch.randn((8, heads, hd), generator=g, device=DEV).bfloat16()
    out, lse = attend(P, c, q, list(range(9)), 1, 8192, 0.125)
    for i in range(8):
        rows = slice(int(c.cu_seq[i]), int(c.cu_seq[i + 1]))
        for h in (0, 17, 63):
            x, y = kk[rows, h].double(), vv[rows, h].double()
            s = x @ q[i, h].double() * 0.125
            w = torch.softmax(s, 0)
            want, mean = w @ y, w @ y.abs()
            size = (x.abs() @ q[i, h].double().abs()).max() * 0.125
            tol = tolerance("bf16", 2.0 ** -16, 0.0, hd, total[i], host(want), host(mean), 0.0, np.asarray(size.item())[None])
            assert np.all(np.abs(host(out[i, h]) - host(want)) <= tol.reshape(-1))
            assert abs(lse[i, h].item() - torch.logsumexp(s, 0).item()) <= lse_tolerance(hd, total[i], lse[i, h].item(), size.item())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_attention_with_holes(P, dtype):
    """Blocks that are not there, requests left out (-1), more rows than tokens (rows that see nothing), longer than max_seq."""
    rng = np.random.default_rng(21)
    total = [50, 40, 3, 20, 64, 30]
    c = Cache(P, rng, total, 2, 64, 16)
    k, v = (randn(rng, (sum(total), 2, 64), "f32") for _ in range(2))
    c.write(P, k, v)
    c.table[0, 1], c.table[0, 2], c.table[3, 0], c.table[3, 1] = c.n_blocks + 5, -1, -9, 2 ** 31 - 1
    c.t_table = i32(c.table)
    seq = [50, -1, 3, 20, 64, 30]
    c.t_seq = i32(seq)
    gone = [np.zeros(64, bool) for _ in total]
    gone[0][16:48] = True
    gone[3][:] = True
    new = [3, 2, 7, 2, 1, 1]
    cu = np.concatenate([[0], np.cumsum(new)])
    q = randn(rng, (int(cu[-1]), 4, 64), dtype)
    for max_q, max_seq in ((32, 1 << 20), (7, 64)):
        out, lse = attend(P, c, q, cu, max_q, max_seq, 0.125)
        check_attend(c, q, out, lse, cu, ref.held(host(k)), ref.held(host(v)), 0.125, dtype, seq=seq, gone=gone)
    assert np.all(host(out)[3:5] == 0) and np.all(np.isneginf(host(lse)[3:5]))
    assert np.all(host(out)[5:9] == 0) and np.all(np.isneginf(host(lse)[5:9]))   # rows 0..3 of 7 with three tokens
    out, lse = attend(P, c, q, cu, 7, 63, 0.125)
    seq[4] = -1
    check_attend(c, q, out, lse, cu, ref.held(host(k)), ref.held(host(v)), 0.125, dtype, seq=seq, gone=gone)
    # rows that make no sense: nothing is written, nothing read out of range
    out, lse = attend(P, c, q, [0, -5, 90, 4, 2, 2 ** 31 - 1, 3], 7, 64, 0.125)
    assert np.all(host(out) == 7)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_attention_with_values_that_are_not_finite(P, dtype):
    """A group that is not finite makes NaN of rows that see it, in its channels only (a key: in all), and of no other row."""
    rng = np.random.default_rng(31)
    total, new = [40, 200, 20, 50], [7, 4, 3, 1]
    c = Cache(P, rng, total, 1, 128, 16)
    k, v = (randn(rng, (sum(total), 1, 128), "f32") for _ in range(2))
    v[36, 0, 40] = math.inf                                            # seen by rows 3.. of 7
    v[40 + 197, 0, 5] = math.nan
    v[40 + 199, 0, 100] = -math.inf
    k[240 + 18, 0, 3] = math.nan                                       # seen by the last two rows
    v[260 + 7, 0, 64] = math.nan
    c.write(P, k, v)
    cu = np.concatenate([[0], np.cumsum(new)])
    q = randn(rng, (int(cu[-1]), 4, 128), dtype)
    for max_q, max_seq in ((32, 1 << 20), (7, 200)):
        out, lse = attend(P, c, q, cu, max_q, max_seq, 0.09)
        with np.errstate(invalid="ignore"):
            check_attend(c, q, out, lse, cu, ref.held(host(k)), ref.held(host(v)), 0.09, dtype)
    assert np.isfinite(host(out)[:3]).all() and np.isnan(host(out)[3:7, :, 32:64]).all() and np.isfinite(host(out)[3:7, :, :32]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rubbish", [0, 253, 254, 255])
def test_attention_with_rubbish_in_unwritten_tokens(P, dtype, rubbish):
    """Blocks whose unwritten tokens hold large exponents and codes of 6 or more."""
    rng = np.random.default_rng(rubbish)
    total = [1, 85, 130, 17]
    for block, hd in ((32, 64), (16, 128)):
        c = Cache(P, rng, total, 2, hd, block)
        c.pool.fill_(rubbish)
        k, v = (randn(rng, (sum(total), 2, hd), "bf16") for _ in range(2))
        c.write(P, k, v)
        q = randn(rng, (8, 4, hd), dtype)
        for max_q, max_seq in ((4, 130), (32, 1 << 20)):
            out, lse = attend(P, c, q, [0, 1, 5, 6, 8], max_q, max_seq, 0.1)
            check_attend(c, q, out, lse, [0, 1, 5, 6, 8], ref.held(host(k)), ref.held(host(v)), 0.1, dtype)


def test_attention_layouts(P):
    """Queries and outputs head-major and inside wider rows."""
    rng = np.random.default_rng(41)
    c = Cache(P, rng, [70, 9], 2, 64, 16)
    k, v = (randn(rng, (79, 2, 64), "bf16") for _ in range(2))
    c.write(P, k, v)
    q = randn(rng, (3, 4, 64), "bf16")
    want, lse = attend(P, c, q, [0, 2, 3], 2, 70, 0.1)
    check_attend(c, q, want, lse, [0, 2, 3], ref.held(host(k)), ref.held(host(v)), 0.1, "bf16")
    q2 = q.transpose(0, 1).contiguous().transpose(0, 1)
    big = torch.full((3, 6, 68), 7.0, dtype=torch.bfloat16, device=DEV)
    out, _ = attend(P, c, q2, [0, 2, 3], 2, 70, 0.1, out=big[:, 1:5, 4:])
    assert torch.equal(out, want)
    out.fill_(7.0)
    assert bool((big == 7).all())


def test_attention_in_a_pool_past_32_bits(P):
    """Blocks whose bytes lie beyond 2^32, slots near the end."""
    block, kv_heads, hd = 64, 8, 128
    n_blocks = (5 << 30) // (block * (hd + hd // 16) * kv_heads)
    pool = torch.empty(P.heisd_kv4_pool_bytes(n_blocks, block, kv_heads, hd), dtype=torch.uint8, device=DEV)
    rng = np.random.default_rng(1)
    c = Cache(P, rng, [100], kv_heads, hd, block)
    c.pool, c.n_blocks, c.desc = pool, n_blocks, P.make_kv4_desc(pool, block, kv_heads, hd)
    c.table[0, :2] = [n_blocks - 1, n_blocks - 7]
    c.t_table = i32(c.table)
    k, v = (randn(rng, (100, kv_heads, hd), "bf16") for _ in range(2))
    c.write(P, k, v)
    gk, gv = c.read(P)
    assert np.array_equal(host(gk), ref.held(host(k))) and np.array_equal(host(gv), ref.held(host(v)))
    q = randn(rng, (1, 8, hd), "bf16")
    out, lse = attend(P, c, q, [0, 1], 1, 100, 0.088)
    check_attend(c, q, out, lse, [0, 1], host(gk), host(gv), 0.088, "bf16")


def prompt(P, q, k, v, cu_q, cu_k, scale, causal, want_lse=True, out=None):
    out = torch.full_like(q, 7.0) if out is None else out
    lse = torch.full(q.shape[:2], 7.0, device=DEV) if want_lse else None
    tq, tk = i32(cu_q), i32(cu_k)
    ok(P, P.heisd_prompt_attention(P.head_rows(q), P.head_rows(k), P.head_rows(v), P.head_rows(out), lse.data_ptr() if want_lse else None,
                                   tq.data_ptr(), tk.data_ptr(), len(cu_q) - 1, q.shape[0], k.shape[0], q.shape[2], scale, int(causal), stream()))
    torch.cuda.synchronize()
    return out, lse


def check_prompt(q, k, v, out, lse, cu_q, cu_k, scale, causal, dtype):
    q64, k64, v64, out = (host(x) for x in (q, k, v, out))
    lse = host(lse) if lse is not None else None
    p, tiny = (2.0 ** -8, 0.0) if dtype == "bf16" else (2.0 ** -11, 2.0 ** -25)
    for i in range(len(cu_q) - 1):
        a, b, n = cu_q[i], cu_q[i + 1], cu_k[i + 1] - cu_k[i]
        kk, vv = k64[cu_k[i]:cu_k[i + 1]], v64[cu_k[i]:cu_k[i + 1]]
        seen = [n - (b - a) + r + 1 if causal else n for r in range(b - a)]
        with np.errstate(invalid="ignore", over="ignore"):
            want, wl, mean, flat, size = ref.attention(q64[a:b], kk, vv, seen, scale)
            odd = ~np.isfinite(want)
            assert np.array_equal(out[a:b][odd], want[odd], equal_nan=True)
            tol = tolerance(dtype, p, tiny, q.shape[2], n, want, mean, flat, size)
            err = np.abs(out[a:b] - want)
        assert np.all((err <= tol)[~odd]), (i, float(np.max((err - tol)[~odd])))
        if lse is None:
            continue
        fine = np.isfinite(wl)
        assert np.array_equal(lse[a:b][~fine], wl[~fine], equal_nan=True)
        assert np.all(np.abs(lse[a:b][fine] - wl[fine]) <= lse_tolerance(q.shape[2], n, wl, size)[fine])


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new,past,heads,head_dim", [
    ([1], [0], (1, 1), 64), ([1, 2, 31, 32, 33], [0, 0, 0, 0, 0], (2, 2), 128), ([127, 128, 129], [0, 5, 64], (4, 1), 64), ([276], [0], (2, 2), 128),
    ([63, 64, 65, 0, 200], [1, 0, 300, 10, 63], (6, 2), 128), ([1, 1, 7], [500, 64, 129], (4, 4), 64), ([300], [200], (5, 1), 128)])
def test_prompt_attention(P, causal, dtype, new, past, heads, head_dim):
    rng = np.random.default_rng(sum(new) + sum(past) + head_dim)
    cu_q, cu_k = np.concatenate([[0], np.cumsum(new)]), np.concatenate([[0], np.cumsum(np.add(new, past))])
    q = randn(rng, (int(cu_q[-1]) + 3, heads[0], head_dim), dtype)
    k, v = (randn(rng, (int(cu_k[-1]) + 2, heads[1], head_dim), dtype) for _ in range(2))
    scale = 1 / math.sqrt(head_dim)
    out, lse = prompt(P, q, k, v, cu_q, cu_k, scale, causal)
    check_prompt(q, k, v, out, lse, cu_q, cu_k, scale, causal, dtype)
    assert np.all(host(out)[cu_q[-1]:] == 7) and np.all(host(lse)[cu_q[-1]:] == 7)
    again, _ = prompt(P, q, k, v, cu_q, cu_k, scale, causal, want_lse=False)
    assert torch.equal(again, out)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("head_dim,causal", [(64, True), (64, False), (128, True), (128, False)])
def test_prompt_attention_of_large_batches(P, dtype, head_dim, causal):
    """A batch with so many (empty) sequences that a workgroup is one set of waves, and the same rows in a small one."""
    rng = np.random.default_rng(head_dim)
    new, past = [129, 1, 300, 0, 70], [0, 333, 64, 5, 500]
    cu_q, cu_k = np.concatenate([[0], np.cumsum(new)]), np.concatenate([[0], np.cumsum(np.add(new, past))])
    q = randn(rng, (500, 4, head_dim), dtype)
    k, v = (randn(rng, (int(cu_k[-1]), 2, head_dim), dtype) for _ in range(2))
    v[129 + 334 + 64 + 290, 0, 1] = math.inf                           # masked for most rows of the third
    for empty in (0, 400):
        a, b = (np.concatenate([x, np.full(empty, x[-1])]) for x in (cu_q, cu_k))
        out, lse = prompt(P, q, k, v, a, b, head_dim ** -0.5, causal)
        check_prompt(q, k, v, out, lse, cu_q, cu_k, head_dim ** -0.5, causal, dtype)


def test_prompt_attention_many_short_sequences(P):
    rng = np.random.default_rng(2)
    new = [int(x) for x in rng.integers(0, 6, 300)]
    past = [int(x) for x in rng.integers(0, 9, 300)]
    cu_q, cu_k = np.concatenate([[0], np.cumsum(new)]), np.concatenate([[0], np.cumsum(np.add(new, past))])
    q = randn(rng, (int(cu_q[-1]), 2, 64), "bf16")
    k, v = (randn(rng, (int(cu_k[-1]), 1, 64), "bf16") for _ in range(2))
    out, lse = prompt(P, q, k, v, cu_q, cu_k, 0.125, True)
    check_prompt(q, k, v, out, lse, cu_q, cu_k, 0.125, True, "bf16")


def test_prompt_attention_rows_that_see_nothing(P):
    """More queries than keys (the first see none), no keys at all, spans that make no sense, and rows of nobody."""
    rng = np.random.default_rng(3)
    cu_q, cu_k = [0, 200, 210, 215], [0, 130, 130, 140]
    q = randn(rng, (220, 2, 128), "bf16")
    k, v = (randn(rng, (140, 1, 128), "bf16") for _ in range(2))
    out, lse = prompt(P, q, k, v, cu_q, cu_k, 0.1, True)
    check_prompt(q, k, v, out, lse, cu_q, cu_k, 0.1, True, "bf16")
    assert np.all(host(out)[:70] == 0) and np.all(np.isneginf(host(lse)[:70])) and np.all(host(out)[200:210] == 0)
    assert np.all(host(out)[215:] == 7)
    out, _ = prompt(P, q, k, v, [0, -1, 500, 2 ** 31 - 1], cu_k, 0.1, True)
    assert np.all(host(out) == 7)
    out, lse = prompt(P, q, k, v, [0, 100, 150, 215], [0, 300, -1, 90], 0.1, True)         # keys that are not there: as if there were none
    assert np.all(host(out)[:215] == 0) and np.all(np.isneginf(host(lse)[:215]))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("head_dim", [64, 128])
def test_prompt_attention_not_finite_where_masked(P, dtype, head_dim):
    """Infinities and NaN in rows that are masked, in other sequences and in rows of nobody have no influence; where they are seen they have
    the plain form's."""
    rng = np.random.default_rng(4)
    new, past = [150, 40, 9], [0, 30, 0]
    cu_q, cu_k = np.concatenate([[0], np.cumsum(new)]), np.concatenate([[0], np.cumsum(np.add(new, past))])
    q = randn(rng, (199, 2, head_dim), dtype)
    k, v = (randn(rng, (int(cu_k[-1]) + 70, 1, head_dim), dtype) for _ in range(2))
    v[100, 0, 3] = math.inf
    v[140, 0, 40] = math.nan
    k[120, 0, 5] = math.nan
    v[150 + 69, 0, 7] = -math.inf                                      # the last token of the second
    k[220:229] = k[220:229] * 0 + 65504 if dtype == "f16" else 3e38
    v[229:], k[229:] = math.nan, math.inf
    out, lse = prompt(P, q, k, v, cu_q, cu_k, 0.1, True)
    check_prompt(q[:190], k, v, out[:190], lse[:190], cu_q[:3], cu_k[:3], 0.1, True, dtype)
    assert np.isfinite(host(out)[:100]).all() and np.isfinite(host(out)[150:189]).all()


@pytest.mark.parametrize("scale", [0.0, -0.2, 1e-42])
def test_attention_with_other_scales(P, scale):
    """Zero (a mean over what is seen), negative and subnormal scales."""
    rng = np.random.default_rng(8)
    q, k, v = (randn(rng, (90, h, 64), "bf16") for h in (2, 1, 1))
    out, lse = prompt(P, q, k, v, [0, 90], [0, 90], scale, True)
    check_prompt(q, k, v, out, lse, [0, 90], [0, 90], scale, True, "bf16")
    c = Cache(P, rng, [90], 1, 64, 16)
    c.write(P, k, v)
    out, lse = attend(P, c, q[:3], [0, 3], 3, 90, scale)
    check_attend(c, q[:3], out, lse, [0, 3], ref.held(host(k)), ref.held(host(v)), scale, "bf16")


def test_prompt_attention_layouts(P):
    rng = np.random.default_rng(5)
    q, k, v = randn(rng, (140, 4, 64), "f16"), randn(rng, (140, 2, 64), "f16"), randn(rng, (140, 2, 64), "f16")
    cu = [0, 140]
    want, lse = prompt(P, q, k, v, cu, cu, 0.125, True)
    check_prompt(q, k, v, want, lse, cu, cu, 0.125, True, "f16")
    fused = torch.cat([q, k, v], 1)                                    # one matrix of rows
    big = torch.full((4, 150, 72), 7.0, dtype=torch.float16, device=DEV)
    out, _ = prompt(P, fused[:, :4], fused[:, 4:6], v.transpose(0, 1).contiguous().transpose(0, 1), cu, cu, 0.125, True,
                    out=big.transpose(0, 1)[5:145, :, 4:68])
    assert torch.equal(out, want)
    out.fill_(7.0)
    assert bool((big == 7).all())


def test_prompt_attention_growing_scores(P):
    """The running maximum moves by more and by less than what is worth rescaling."""
    rng = np.random.default_rng(6)
    n = 700
    q, v = randn(rng, (n, 1, 128), "bf16"), randn(rng, (n, 1, 128), "bf16")
    for step in (0.005, 0.05, -0.05):
        k = (torch.arange(n, device=DEV)[:, None, None] * step * torch.sign(q[-1].float())[None] / 4 + randn(rng, (n, 1, 128), "f32") * 0.1).to(torch.bfloat16)
        out, lse = prompt(P, q, k, v, [0, n], [0, n], 0.088, True)
        check_prompt(q, k, v, out, lse, [0, n], [0, n], 0.088, True, "bf16")
