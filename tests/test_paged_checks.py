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
