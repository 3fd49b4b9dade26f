"""Requests that continue others where the calls meet each other: groups that describe nothing beside those that do, evictions between other calls, bounds that
differ, the exactness of attention over prefixes of many rows.  Tolerances: those of test_gpu_branch.py, except where a test derives its own."""
import numpy as np
import pytest

import paged_reference as ref

torch = pytest.importorskip("torch")
from test_gpu_branch import WIDE, prefix_of, shared  # noqa: E402
from test_gpu_paged import Cache, host, randn, tolerance  # noqa: E402

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
