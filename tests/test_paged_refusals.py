"""What the calls on paged requests refuse before they touch a device, and their host-side results (no GPU)."""
import ctypes
import math

import numpy as np
import pytest

import paged_reference as ref

FAKE = 0x10000      # never dereferenced: every check below fails before any device access


@pytest.fixture(scope="module")
def P():
    import paper_2603_17573_amd as P
    from paper_2603_17573_amd import binding, build
    import os
    if not os.path.exists(binding.LIB_PATH):
        build.build(force=False)
    return P


def rows(P, data=FAKE, rs=1024, hs=128, heads=8, dtype=0):
    return P.heisd_head_rows(data, rs, hs, heads, dtype)


def refused(P, rc, code, *words):
    assert rc == code, (rc, P.heisd_last_error(None))
    text = P.heisd_last_error(None)
    for w in words:
        assert w in text, text


def plan_desc(P, **more):
    d = P.heisd_plan_desc(4, 16, 8, 64, 20)
    for n, _ in P.heisd_plan_desc._fields_[5:]:
        setattr(d, n, FAKE)
    for k, v in more.items():
        setattr(d, k, v)
    return d


def test_struct_layouts(P):
    assert ctypes.sizeof(P.heisd_head_rows) == 32 and ctypes.sizeof(P.heisd_kv4_desc) == 24
    assert ctypes.sizeof(P.heisd_paged_batch) == 40 and ctypes.sizeof(P.heisd_rope_desc) == 64
    assert P.heisd_plan_desc.cached_len.offset == 24 and ctypes.sizeof(P.heisd_plan_desc) == 24 + 13 * 8


def test_plan_refusals(P):
    refused(P, P.heisd_paged_plan(None, None), P.HEISD_EINVAL, "NULL")
    for more in (dict(batch=0), dict(batch=65536), dict(rows=-1), dict(rows=(1 << 30) + 1), dict(block_size=0), dict(n_blocks=0), dict(max_blocks=0),
                 dict(max_blocks=(1 << 20) + 1), dict(n_blocks=1 << 28, block_size=16), dict(max_blocks=1 << 20, block_size=4096, n_blocks=1)):
        refused(P, P.heisd_paged_plan(plan_desc(P, **more), None), P.HEISD_EINVAL, "paged_plan")
    for n, _ in P.heisd_plan_desc._fields_[5:]:
        if n != "cu_seq":
            refused(P, P.heisd_paged_plan(plan_desc(P, **{n: None}), None), P.HEISD_EINVAL, "NULL")


def test_rope_table_refusals_and_values(P):
    table = lambda *a, **k: P.heisd_rope_table(P.make_rope_desc(*a, **k))  # noqa: E731
    for a in ((0,), (3,), (258,), (64, 1.0), (64, math.inf), (64, math.nan)):
        refused(P, table(*a)[0], P.HEISD_EINVAL, "rope_table")
    for k in (dict(scaling="linear", factor=0.5), dict(scaling="base", factor=math.nan), dict(scaling="parts", factor=2.0),
              dict(scaling="parts", factor=2.0, original_len=10, beta_fast=1.0), dict(scaling="bands", factor=2.0, original_len=10, low_freq=4.0),
              dict(scaling="bands", factor=2.0, original_len=0)):
        refused(P, table(64, **k)[0], P.HEISD_EINVAL, "rope_table")
    d = P.make_rope_desc(64)
    d.scaling = 9
    refused(P, P.heisd_rope_table(d)[0], P.HEISD_EINVAL, "scaling")
    for n in (2, 20, 64, 128, 256):
        for scaling in ("none", "linear", "base", "parts", "bands"):
            more = dict(factor=4.0, original_len=2048) if scaling != "none" else {}
            rc, turns, size = table(n, 50000.0, scaling, **more)
            freq, want = ref.frequencies(n, 50000.0, scaling, more.get("factor", 1.0), more.get("original_len", 0))
            # a dozen 64-bit operations, each to 2^-52
            assert rc == 0 and np.abs(np.array(turns) * 2 * math.pi - freq).max() <= 1e-13 and abs(size - want) <= 2.0 ** -23
            assert np.all(np.abs(np.array(turns) * 2 * math.pi / freq - 1) <= 1e-13)


def test_rope_refusals(P):
    def rope(turns=FAKE, size=1.0, rotary=64, layout=0, position=FAKE, n=5, head_dim=128, q=None, qo=None, k=None, ko=None):
        q, qo = q or rows(P), qo or rows(P, 0x20000)
        return P.heisd_rope(turns, size, rotary, layout, 0, position, n, head_dim, q, qo, k, ko, None)
    for more in (dict(turns=None), dict(turns=FAKE + 4), dict(size=math.nan), dict(rotary=0), dict(rotary=63), dict(rotary=130), dict(layout=2),
                 dict(position=None), dict(n=-1), dict(head_dim=257), dict(head_dim=1), dict(k=rows(P)), dict(ko=rows(P)), dict(q=rows(P, 0)),
                 dict(q=rows(P, dtype=3)), dict(q=rows(P, dtype=2)), dict(q=rows(P, heads=4)), dict(qo=rows(P, heads=0)), dict(q=rows(P, heads=513), qo=rows(P, heads=513)),
                 dict(q=rows(P, FAKE + 1)), dict(qo=rows(P, rs=2048)), dict(k=rows(P), ko=rows(P, 0x30000, heads=4)), dict(q=rows(P, rs=-8)), dict(qo=rows(P, 0x20000, hs=-1))):
        refused(P, rope(**more), P.HEISD_EINVAL, "rope")
    assert rope(n=0) == P.HEISD_OK


def test_cache_refusals(P):
    assert P.heisd_kv4_pool_bytes(10, 16, 8, 128) == 10 * 8 * 16 * 136
    for a in ((0, 16, 8, 128), (10, 24, 8, 128), (10, 8, 8, 128), (10, 8192, 8, 128), (10, 16, 0, 128), (10, 16, 513, 128), (10, 16, 8, 96), (1 << 28, 16, 1, 64)):
        assert P.heisd_kv4_pool_bytes(*a) == 0
    good = P.heisd_kv4_desc(FAKE, 10, 16, 8, 128)
    slot = 0x40000
    bad = [(P.heisd_kv4_desc(0, 10, 16, 8, 128), P.HEISD_EINVAL), (P.heisd_kv4_desc(FAKE + 8, 10, 16, 8, 128), P.HEISD_EINVAL),
           (P.heisd_kv4_desc(FAKE, 10, 24, 8, 128), P.HEISD_EINVAL), (P.heisd_kv4_desc(FAKE, 0, 16, 8, 128), P.HEISD_EINVAL),
           (P.heisd_kv4_desc(FAKE, 10, 16, 8, 80), P.HEISD_EUNSUPPORTED), (None, P.HEISD_EINVAL)]
    b = P.heisd_paged_batch(FAKE, FAKE, FAKE, 2, 4, 6)
    for c, code in bad:
        refused(P, P.heisd_kv4_append(c, rows(P), rows(P), slot, 4, None), code, "kv4_append")
        refused(P, P.heisd_kv4_gather(c, b, FAKE, 4, rows(P), rows(P), None), code, "kv4_gather")
        refused(P, P.heisd_kv4_attention(c, b, rows(P), rows(P), None, 0.1, 1, 64, FAKE, 1 << 20, None), code, "kv4_attention")
        assert P.heisd_kv4_attention_workspace_bytes(c, 2, 6, 8, 1, 64) == 0 or c is not None and c.pool != FAKE
    for k, v in ((None, rows(P)), (rows(P), None), (rows(P, heads=4), rows(P)), (rows(P, dtype=1), rows(P)), (rows(P), rows(P, FAKE + 1)), (rows(P, hs=-128), rows(P))):
        refused(P, P.heisd_kv4_append(good, k, v, slot, 4, None), P.HEISD_EINVAL)
        refused(P, P.heisd_kv4_gather(good, b, FAKE, 4, k, v, None), P.HEISD_EINVAL)
    refused(P, P.heisd_kv4_append(good, rows(P), rows(P), None, 4, None), P.HEISD_EINVAL)
    refused(P, P.heisd_kv4_append(good, rows(P), rows(P), slot, -4, None), P.HEISD_EINVAL)
    refused(P, P.heisd_kv4_gather(good, b, None, 4, rows(P), rows(P), None), P.HEISD_EINVAL)
    refused(P, P.heisd_kv4_gather(good, b, FAKE, -1, rows(P), rows(P), None), P.HEISD_EINVAL)
    assert P.heisd_kv4_append(good, rows(P), rows(P), None, 0, None) == 0 and P.heisd_kv4_gather(good, b, FAKE, 0, rows(P), rows(P), None) == 0


def test_attention_refusals(P):
    c = P.heisd_kv4_desc(FAKE, 10, 16, 2, 128)
    ws = P.heisd_kv4_attention_workspace_bytes(c, 2, 6, 8, 3, 4000)
    assert ws > 256

    def call(b=None, q=None, out=None, scale=0.1, max_q=3, max_seq=4000, workspace=FAKE, n=None, **batch):
        b = b or P.heisd_paged_batch(*[batch.get(k, d) for k, d in (("table", FAKE), ("seq", FAKE), ("cu", FAKE), ("batch", 2), ("max_blocks", 4), ("rows", 6))])
        return P.heisd_kv4_attention(c, b, q or rows(P), out or rows(P, 0x20000), None, scale, max_q, max_seq, workspace, ws if n is None else n, None)
    for more in (dict(table=None), dict(seq=None), dict(cu=None), dict(batch=0), dict(batch=65536), dict(max_blocks=0), dict(rows=-1), dict(scale=math.inf), dict(max_q=0),
                 dict(max_seq=0), dict(max_seq=(1 << 24) + 1), dict(workspace=None), dict(workspace=FAKE + 16), dict(q=rows(P, heads=7)), dict(q=rows(P, heads=4)),
                 dict(out=rows(P, dtype=1)), dict(q=rows(P, FAKE + 8)), dict(q=rows(P, rs=1028)), dict(out=rows(P, hs=130)), dict(q=rows(P, 0))):
        refused(P, call(**more), P.HEISD_EINVAL, "kv4_attention")
    refused(P, call(q=rows(P, dtype=2), out=rows(P, dtype=2)), P.HEISD_EUNSUPPORTED, "fp32")
    refused(P, call(n=ws - 1), P.HEISD_ENOMEM, "workspace")
    refused(P, P.heisd_kv4_attention(c, None, rows(P), rows(P), None, 0.1, 1, 64, FAKE, 1 << 20, None), P.HEISD_EINVAL)
    assert call(rows=0) == P.HEISD_OK
    for a in ((0, 6, 8, 3, 100), (2, -1, 8, 3, 100), (2, 6, 7, 3, 100), (2, 6, 8, 0, 100), (2, 6, 8, 3, 0), (2, 6, 1024, 3, 100)):
        assert P.heisd_kv4_attention_workspace_bytes(c, *a) == 0


def test_prompt_refusals(P):
    def call(q=None, k=None, v=None, out=None, cu_q=FAKE, cu_k=FAKE, batch=2, n=10, kn=10, head_dim=128, scale=0.1):
        return P.heisd_prompt_attention(q or rows(P), k or rows(P, heads=2), v or rows(P, heads=2), out or rows(P, 0x20000), None, cu_q, cu_k, batch, n, kn, head_dim, scale, 1,
                                        None)
    for more in (dict(cu_q=None), dict(cu_k=None), dict(batch=0), dict(batch=65536), dict(n=-1), dict(kn=-1), dict(scale=math.nan), dict(q=rows(P, heads=7)),
                 dict(k=rows(P, heads=3)), dict(v=rows(P, heads=4)), dict(out=rows(P, heads=4)), dict(k=rows(P, heads=2, dtype=1)), dict(out=rows(P, dtype=1)),
                 dict(q=rows(P, FAKE + 8)), dict(k=rows(P, heads=2, rs=1028)), dict(v=rows(P, heads=2, hs=4)), dict(out=rows(P, FAKE + 2)), dict(q=rows(P, 0)),
                 dict(k=rows(P, 0, heads=2)), dict(q=rows(P, dtype=5))):
        refused(P, call(**more), P.HEISD_EINVAL, "prompt_attention")
    f32 = rows(P, dtype=2)
    refused(P, call(q=f32, k=rows(P, heads=2, dtype=2), v=rows(P, heads=2, dtype=2), out=f32), P.HEISD_EUNSUPPORTED, "fp32")
    refused(P, call(head_dim=96), P.HEISD_EUNSUPPORTED, "head_dim")
    for more in (dict(k=rows(P, heads=2, rs=(1 << 25) + 8)), dict(v=rows(P, heads=2, rs=1 << 40))):
        refused(P, call(**more), P.HEISD_EUNSUPPORTED, "apart")
    assert call(n=0) == P.HEISD_OK


def test_torch_side_checks(P):
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    assert P.head_rows(x).row_stride == 128 and P.head_rows(x.transpose(0, 1)).heads == 4
    for bad in (x[0], x.double(), x[..., ::2]):
        with pytest.raises(ValueError):
            P.head_rows(bad)
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        P.make_paged_batch(torch.zeros(3, 4, dtype=torch.int64), i, i, 1)
    with pytest.raises(ValueError):
        P.make_paged_batch(torch.zeros(3, 4, dtype=torch.int32), i, i, 1)
    with pytest.raises(ValueError):
        P.make_kv4_desc(torch.zeros(100, dtype=torch.uint8), 16, 1, 64)
    with pytest.raises(ValueError):
        P.rope_table(P.make_rope_desc(63), "cpu")


def test_the_two_references_of_the_format_agree():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((40, 3, 64)) * np.exp(4 * rng.standard_normal((40, 3, 1)))
    x[0, 0, :32] = 0
    x[1, 0, :32] = [0.25, -0.75, 1.25, 1.75, -2.5, 3.5, 5, 6] * 4
    x[2, 0, :32] = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -6.0001] * 4) * 2.0 ** -130
    x[3, 1, 40], x[3, 2, 0] = np.inf, np.nan
    x[4, 0, 5] = 3 * 2.0 ** 127
    assert np.array_equal(ref.held(x), ref.held_plain(x), equal_nan=True)
    assert np.array_equal(np.signbit(ref.held(x[:3])), np.signbit(ref.held_plain(x[:3])))
