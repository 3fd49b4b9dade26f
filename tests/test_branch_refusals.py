"""What the calls on requests that continue others refuse on the host (no GPU): every check comes before any device access."""
import ctypes

import pytest

FAKE = 0x10000      # never dereferenced: every call below ends before any device access


@pytest.fixture(scope="module")
def P():
    import os
    import paper_2603_17573_amd as P
    from paper_2603_17573_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build(force=False)
    return P


def refused(P, rc, code, *words):
    assert rc == code, (rc, P.heisd_last_error(None))
    text = P.heisd_last_error(None)
    for w in words:
        assert w in text, text


def fill(desc, start, **more):
    for n, t in desc._fields_[start:]:
        if t is ctypes.c_void_p:
            setattr(desc, n, FAKE + 0x1000 * (1 + [f[0] for f in desc._fields_].index(n)))
    for k, v in more.items():
        setattr(desc, k, v)
    return desc


def test_struct_layouts(P):
    assert ctypes.sizeof(P.heisd_beam_desc) == 8 + 8 + 6 * 4 + 8 + 9 * 8 + 8
    assert P.heisd_beam_desc.length_power.offset == 40 and P.heisd_beam_desc.first.offset == 120
    assert ctypes.sizeof(P.heisd_reorder_desc) == 24 + 11 * 8 and P.heisd_reorder_desc.parent.offset == 24
    assert ctypes.sizeof(P.heisd_prefix_groups) == 32


def beams(P, **more):
    return fill(P.heisd_beam_desc(FAKE, 100, 2, 3, 4, 4, 100, 7, 0.5), 9, **{"first": 0, "stride": 4, **more})


def test_beam_select(P):
    n = P.heisd_beam_select_workspace_bytes(3, 4, 4, 100)
    assert n > 0 and P.heisd_beam_select_workspace_bytes(1, 64, 64, 524280) > 0
    for bad in ((0, 4, 4, 100), (65536, 1, 1, 100), (1, 65, 4, 100), (1, 4, 65, 100), (1, 0, 4, 100), (1, 4, 0, 100), (1, 4, 4, 0), (1, 4, 4, 524281), (2000, 64, 4, 100)):
        assert P.heisd_beam_select_workspace_bytes(*bad) == 0
    for more in (dict(logits=None), dict(logits=FAKE + 2), dict(row_stride=-1), dict(dtype=3), dict(groups=0), dict(beams=65), dict(width=0), dict(vocab=0), dict(score_in=None),
                 dict(score_out=None), dict(beam=None), dict(token=None), dict(length_out=None), dict(length_in=None), dict(done_in=None), dict(done_out=None),
                 dict(end_token=100), dict(end_token=-2), dict(length_power=float("nan")), dict(length_power=float("inf")), dict(first=-1), dict(stride=3),
                 dict(first=2 ** 31 - 5), dict(length_in=None, length_out=None), dict(done_in=None, done_out=None), dict(score_out=beams(P).score_in, width=3)):
        refused(P, P.heisd_beam_select(beams(P, **more), FAKE, n, None), P.HEISD_EINVAL, "beam_select")
    refused(P, P.heisd_beam_select(None, FAKE, n, None), P.HEISD_EINVAL, "NULL")
    refused(P, P.heisd_beam_select(beams(P), None, n, None), P.HEISD_EINVAL, "workspace")
    refused(P, P.heisd_beam_select(beams(P), FAKE + 16, n, None), P.HEISD_EINVAL, "workspace")
    refused(P, P.heisd_beam_select(beams(P), FAKE, 0, None), P.HEISD_ENOMEM, "workspace")


def reorder(P, **more):
    return fill(P.heisd_reorder_desc(4, 16, 8, 64, 0), 5, **more)


def test_paged_reorder(P):
    names = [n for n, _ in P.heisd_reorder_desc._fields_[5:]]
    for more in [{n: None} for n in names] + [dict(batch=0), dict(batch=65536), dict(block_size=0), dict(n_blocks=0), dict(max_blocks=0), dict(max_blocks=(1 << 20) + 1),
                                              dict(n_blocks=1 << 28), dict(max_blocks=1 << 20, block_size=4096), dict(len_out=reorder(P).len_in),
                                              dict(owned_out=reorder(P).owned_in), dict(table_out=reorder(P).table_in),
                                              dict(len_out=reorder(P).parent), dict(copy_from=reorder(P).parent), dict(copy_from=reorder(P).len_in)]:
        refused(P, P.heisd_paged_reorder(reorder(P, **more), None), P.HEISD_EINVAL, "paged_reorder")
    refused(P, P.heisd_paged_reorder(None, None), P.HEISD_EINVAL, "NULL")


def cache(P, **more):
    return P.heisd_kv4_desc(more.get("pool", FAKE), more.get("n_blocks", 8), more.get("block_size", 16), more.get("kv_heads", 2), more.get("head_dim", 128))


def batch(P, **more):
    return P.heisd_paged_batch(*[more.get(n, x) for n, x in (("table", FAKE), ("seq", 0x20000), ("cu", FAKE), ("batch", 2), ("max_blocks", 4), ("rows", 6))])


def rows(P, data=FAKE, rs=1024, hs=128, heads=8, dtype=0):
    return P.heisd_head_rows(data, rs, hs, heads, dtype)


def groups(P, **more):
    return P.heisd_prefix_groups(more.get("first", FAKE), more.get("prefix", FAKE), more.get("groups", 2), more.get("max_rows", 3), more.get("max_prefix", 60))


BAD_CACHE = (dict(pool=None), dict(pool=FAKE + 8), dict(n_blocks=0), dict(block_size=24), dict(kv_heads=0))
BAD_BATCH = (dict(table=None), dict(seq=None), dict(batch=0), dict(batch=65536), dict(max_blocks=0), dict(rows=-1))


def test_layers(P):
    size = P.heisd_kv4_pool_bytes(8, 16, 2, 128)

    def copy(c=None, layers=2, apart=size, b=None, source=FAKE, most=64):
        return P.heisd_kv4_copy(c or cache(P), layers, apart, b or batch(P), source, None, most, None)

    def evict(c=None, layers=2, apart=size, b=None, keep=FAKE, recent=3, w=FAKE, out=FAKE, seq=0x30000, most=64):
        return P.heisd_kv4_evict(c or cache(P), layers, apart, b or batch(P), keep, recent, w, out, seq, most, None)
    for call, who in ((copy, "kv4_copy"), (evict, "kv4_evict")):
        for kw in [dict(c=cache(P, **m)) for m in BAD_CACHE] + [dict(b=batch(P, **m)) for m in BAD_BATCH] + \
                [dict(layers=0), dict(layers=65536), dict(apart=size - 16), dict(apart=size + 8), dict(most=0)]:
            refused(P, call(**kw), P.HEISD_EINVAL, who)
        refused(P, call(c=cache(P, head_dim=96)), P.HEISD_EUNSUPPORTED, "head_dim")
    refused(P, copy(source=None), P.HEISD_EINVAL, "NULL")
    for kw in (dict(keep=None), dict(w=None), dict(out=None), dict(seq=None), dict(recent=-1), dict(most=(1 << 24) + 1), dict(seq=0x20000), dict(seq=FAKE)):
        refused(P, evict(**kw), P.HEISD_EINVAL, "kv4_evict")


def test_shared_attention(P):
    n = P.heisd_kv4_shared_attention_workspace_bytes(cache(P), 2, 6, 8, 3, 64, groups(P))
    assert n > 0 and P.heisd_kv4_shared_attention_workspace_bytes(cache(P), 2, 6, 8, 3, 64, None) > 0
    bad = (dict(groups=-1), dict(groups=65536), dict(max_rows=0), dict(max_prefix=0), dict(max_prefix=(1 << 24) + 1), dict(first=None), dict(prefix=None))
    for more in bad:
        assert P.heisd_kv4_shared_attention_workspace_bytes(cache(P), 2, 6, 8, 3, 64, groups(P, **more)) == 0
    assert P.heisd_kv4_shared_attention_workspace_bytes(cache(P), 2, 6, 7, 3, 64, groups(P)) == 0
    assert P.heisd_kv4_shared_attention_workspace_bytes(cache(P), 0, 6, 8, 3, 64, groups(P)) == 0

    def call(c=None, b=None, g=None, q=None, out=None, scale=0.1, max_q=3, most=64, ws=FAKE, size=n):
        return P.heisd_kv4_shared_attention(c or cache(P), b or batch(P), g or groups(P), q or rows(P), out or rows(P, 0x20000), None, scale, max_q, most, ws, size, None)
    for kw in [dict(c=cache(P, **m)) for m in BAD_CACHE] + [dict(b=batch(P, **m)) for m in BAD_BATCH + (dict(cu=None),)] + [dict(g=groups(P, **m)) for m in bad] + \
            [dict(q=rows(P, heads=7)), dict(q=rows(P, dtype=1)), dict(q=rows(P, FAKE + 8)), dict(out=rows(P, FAKE + 2)), dict(out=rows(P, rs=64)), dict(out=rows(P, hs=0)),
             dict(q=rows(P, None)), dict(scale=float("nan")), dict(max_q=0), dict(most=0), dict(most=(1 << 24) + 1), dict(ws=None), dict(ws=FAKE + 128)]:
        refused(P, call(**kw), P.HEISD_EINVAL, "kv4_shared_attention")
    refused(P, call(c=cache(P, head_dim=96)), P.HEISD_EUNSUPPORTED, "head_dim")
    refused(P, call(q=rows(P, dtype=2), out=rows(P, dtype=2)), P.HEISD_EUNSUPPORTED, "fp32")
    refused(P, call(size=n - 1), P.HEISD_ENOMEM, "workspace")
    assert call(b=batch(P, rows=0)) == 0


def test_weigh_and_offset(P):
    def call(c=None, b=None, g=None, q=None, lse=FAKE, scale=0.1, decay=1.0, w=FAKE, out=FAKE, most=64):
        return P.heisd_kv4_weigh(c or cache(P), b or batch(P), g or groups(P), q or rows(P), lse, scale, decay, w, out, most, None)
    for kw in [dict(c=cache(P, **m)) for m in BAD_CACHE] + [dict(b=batch(P, **m)) for m in BAD_BATCH + (dict(cu=None),)] + \
            [dict(q=rows(P, heads=7)), dict(q=rows(P, FAKE + 8)), dict(q=rows(P, None)), dict(lse=None), dict(w=None), dict(out=None), dict(scale=float("inf")),
             dict(decay=float("nan")), dict(most=0), dict(most=(1 << 24) + 1), dict(g=groups(P, max_prefix=0))]:
        refused(P, call(**kw), P.HEISD_EINVAL, "kv4_weigh")
    refused(P, call(q=rows(P, dtype=2)), P.HEISD_EUNSUPPORTED, "fp32")
    for b in BAD_BATCH + (dict(cu=None),):
        refused(P, P.heisd_paged_offset(batch(P, **b), FAKE, FAKE, None), P.HEISD_EINVAL, "paged_offset")
    refused(P, P.heisd_paged_offset(batch(P), None, FAKE, None), P.HEISD_EINVAL, "NULL")
    refused(P, P.heisd_paged_offset(batch(P), FAKE, None, None), P.HEISD_EINVAL, "NULL")
    assert P.heisd_paged_offset(batch(P, rows=0), FAKE, None, None) == 0
