"""What the calls on paged requests refuse on the host, beyond test_paged_refusals.py (no GPU): tensors that are not where the kernels
would look for them, outputs whose rows lie on each other, sizes past what a launch or 64-bit arithmetic holds."""
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def P():
    import os
    import paper_2603_17573_amd as P
    from paper_2603_17573_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build(force=False)
    return P


def test_host_tensors_are_refused(P):
    """Of the right type and shape, but in host memory: a kernel would take their addresses for its own."""
    def i(*shape):
        return torch.zeros(shape, dtype=torch.int32)
    with pytest.raises(ValueError, match="on a GPU"):
        P.make_plan_desc(16, 8, i(2), i(2), i(2), i(2), i(2, 4), i(8), i(1), i(1), i(2), i(3), i(5), i(5), i(3))
    with pytest.raises(ValueError, match="on a GPU"):
        P.make_paged_batch(i(2, 4), i(2), i(3), 5)
    with pytest.raises(ValueError, match="on a GPU"):
        P.make_paged_batch(i(2, 4), i(2), None, 0)
    with pytest.raises(ValueError, match="on a GPU"):
        P.make_kv4_desc(torch.zeros(16 * 68, dtype=torch.uint8), 16, 1, 64)


def test_a_cache_of_no_tokens_per_block_is_refused(P):
    for size in (0, -16, 24):
        with pytest.raises(ValueError, match="invalid cache"):
            P.PagedCache(1, 2, 1, 64, 2, 200, 300, n_blocks=8, block_size=size)


FAKE = 0x10000      # never dereferenced: every call below ends before any device access


def rows(P, data=FAKE, rs=1024, hs=128, heads=8, dtype=0):
    return P.heisd_head_rows(data, rs, hs, heads, dtype)


def refused(P, rc, code, *words):
    assert rc == code, (rc, P.heisd_last_error(None))
    text = P.heisd_last_error(None)
    for w in words:
        assert w in text, text


def test_paged_prompt_refusals(P):
    def call(q=None, k=None, v=None, out=None, head_dim=128, scale=0.1, **b):
        desc = P.heisd_paged_batch(*[b.get(n, x) for n, x in (("table", FAKE), ("seq", FAKE), ("cu", FAKE), ("batch", 2), ("max_blocks", 4), ("rows", 6))])
        return P.heisd_paged_prompt_attention(desc, q or rows(P), k or rows(P, heads=2), v or rows(P, heads=2), out or rows(P, 0x20000), None, head_dim, scale, None)
    for more in (dict(table=None), dict(seq=None), dict(cu=None), dict(batch=0), dict(batch=65536), dict(rows=-1), dict(scale=float("nan")), dict(q=rows(P, heads=7)),
                 dict(k=rows(P, heads=2, dtype=1)), dict(v=rows(P, heads=4)), dict(q=rows(P, FAKE + 8)), dict(out=rows(P, FAKE + 2)), dict(q=rows(P, 0))):
        refused(P, call(**more), P.HEISD_EINVAL, "paged_prompt_attention")
    refused(P, call(head_dim=96), P.HEISD_EUNSUPPORTED, "head_dim")
    refused(P, P.heisd_paged_prompt_attention(None, rows(P), rows(P), rows(P), rows(P), None, 128, 0.1, None), P.HEISD_EINVAL, "NULL")
    assert call(rows=0) == P.HEISD_OK


def test_rows_that_there_are_none_of_need_no_memory(P):
    """What an empty tensor gives: NULL."""
    none, one = rows(P, 0), rows(P, 0, heads=2)
    cache, slot = P.heisd_kv4_desc(FAKE, 10, 16, 8, 128), None
    assert P.heisd_rope(FAKE, 1.0, 64, 0, 0, None, 0, 128, none, none, one, one, None) == P.HEISD_OK
    assert P.heisd_kv4_append(cache, none, none, slot, 0, None) == P.HEISD_OK
    b = P.heisd_paged_batch(FAKE, FAKE, FAKE, 2, 4, 0)
    assert P.heisd_kv4_gather(cache, b, FAKE, 0, none, none, None) == P.HEISD_OK
    assert P.heisd_kv4_attention(cache, b, none, none, None, 0.1, 1, 64, FAKE, 0, None) == P.HEISD_OK
    assert P.heisd_prompt_attention(none, one, one, none, None, FAKE, FAKE, 2, 0, 0, 128, 0.1, 1, None) == P.HEISD_OK
    assert P.heisd_paged_prompt_attention(b, none, one, one, none, None, 128, 0.1, None) == P.HEISD_OK
    # what there is must lie somewhere
    refused(P, P.heisd_rope(FAKE, 1.0, 64, 0, 0, FAKE, 1, 128, none, none, None, None, None), P.HEISD_EINVAL, "NULL q")
    refused(P, P.heisd_prompt_attention(rows(P), one, one, rows(P), None, FAKE, FAKE, 2, 4, 1, 128, 0.1, 1, None), P.HEISD_EINVAL, "NULL k")
    refused(P, P.heisd_prompt_attention(none, one, one, none, None, FAKE, FAKE, 2, 4, 0, 128, 0.1, 1, None), P.HEISD_EINVAL, "NULL q")
    refused(P, P.heisd_kv4_append(cache, none, none, FAKE, -1, None), P.HEISD_EINVAL, "rows=-1")


def test_more_rows_than_a_launch_takes(P):
    """2^32 threads or more in one direction of a grid, and counts next to the end of 32 bits."""
    most, cache = 2 ** 31 - 1, P.heisd_kv4_desc(FAKE, 10, 16, 8, 128)
    for heads, dim, n in ((1, 256, most), (1, 256, 2 ** 25), (8, 64, most)):      # 256 / pairs rows per workgroup
        q = rows(P, rs=heads * dim, hs=dim, heads=heads)
        refused(P, P.heisd_rope(FAKE, 1.0, dim, 0, 0, FAKE, n, dim, q, q, None, None, None), P.HEISD_EINVAL, "too many rows")
    for heads, n in ((512, most), (512, 2 ** 24), (16, most), (16, 2 ** 28)):
        c, k = P.heisd_kv4_desc(FAKE, 10, 16, heads, 128), rows(P, heads=heads)
        refused(P, P.heisd_kv4_append(c, k, k, FAKE, n, None), P.HEISD_EINVAL, "too many rows")
    b = P.heisd_paged_batch(FAKE, FAKE, FAKE, 2, 4, 6)
    for dtype, n in ((0, most), (0, 2 ** 28), (2, 2 ** 27)):
        k = rows(P, dtype=dtype)
        refused(P, P.heisd_kv4_gather(cache, b, FAKE, n, k, k, None), P.HEISD_EINVAL, "too many rows")
    for heads, batch, n in ((512, 1, 2 ** 22), (512, 65535, 1), (2, 1, most), (1, 1, most)):
        q = rows(P, heads=heads)
        refused(P, P.heisd_prompt_attention(q, q, q, q, None, FAKE, FAKE, batch, n, n, 128, 0.1, 1, None), P.HEISD_EINVAL, "too many rows")


def test_outputs_on_each_other_are_refused(P):
    """What a broadcast or overlapping view gives; inputs may be broadcast."""
    cache, b = P.heisd_kv4_desc(FAKE, 10, 16, 8, 128), P.heisd_paged_batch(FAKE, FAKE, FAKE, 2, 4, 6)
    good, ws = rows(P, 0x20000), P.heisd_kv4_attention_workspace_bytes(cache, 2, 6, 8, 1, 64)
    for bad in (rows(P, rs=0), rows(P, hs=0), rows(P, hs=64), rows(P, rs=120, hs=1024), rows(P, rs=0, hs=0)):
        refused(P, P.heisd_rope(FAKE, 1.0, 64, 0, 0, FAKE, 6, 128, bad, bad, None, None, None), P.HEISD_EINVAL, "q_out lie on each other")
        refused(P, P.heisd_rope(FAKE, 1.0, 64, 0, 0, FAKE, 6, 128, good, good, bad, bad, None), P.HEISD_EINVAL, "k_out lie on each other")
        refused(P, P.heisd_kv4_gather(cache, b, FAKE, 6, bad, good, None), P.HEISD_EINVAL, "k_out lie on each other")
        refused(P, P.heisd_kv4_gather(cache, b, FAKE, 6, good, bad, None), P.HEISD_EINVAL, "v_out lie on each other")
        refused(P, P.heisd_kv4_attention(cache, b, good, bad, None, 0.1, 1, 64, FAKE, ws, None), P.HEISD_EINVAL, "out lie on each other")
        refused(P, P.heisd_prompt_attention(good, good, good, bad, None, FAKE, FAKE, 2, 6, 6, 128, 0.1, 1, None), P.HEISD_EINVAL, "out lie on each other")
        refused(P, P.heisd_paged_prompt_attention(b, good, good, good, bad, None, 128, 0.1, None), P.HEISD_EINVAL, "out lie on each other")


def test_bounds_at_their_largest_do_not_wrap(P):
    """Workspaces do not shrink where the bounds grow, up to the largest that are taken: 65535 requests, 512 key heads, 2^31 - 1 rows, 2^24
    tokens, whose product passes 64 bits."""
    for heads in (1, 512):
        cache, last = P.heisd_kv4_desc(FAKE, 10, 16, heads, 128), 0
        for max_q in (1, 33, 1 << 10, 1 << 20, 1 << 27, 1 << 30, 2 ** 31 - 1):
            n = P.heisd_kv4_attention_workspace_bytes(cache, 65535, 6, 512, max_q, 1 << 24)
            assert n > 0 and n >= last, (heads, max_q, n, last)
            last = n
        # as many workgroups and columns as there ever are
        assert last == P.heisd_kv4_attention_workspace_bytes(cache, 65535, 6, 512, 64, 1 << 24)
