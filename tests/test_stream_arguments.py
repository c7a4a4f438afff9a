"""Arguments of the binding that are refused on the host."""
import pytest

from paper_2608_26965_b200 import binding, build


@pytest.mark.parametrize("big", [2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 63 - 1, -2 ** 31 - 1, -2 ** 32])
def test_numbers_beyond_32_bits_are_refused(big):
    """Taken modulo 2^32 a bound of 2^32 rows would be one of none."""
    window = dict(batch=1, heads_q=1, heads_kv=1, n_q=4, n_k=4, head_dim=64, dtype="bf16", left=1, right=0, sinks=0, flags=0)
    cache = dict(batch=1, heads_q=1, heads_kv=1, head_dim=64, dtype="bf16", page_rows=16, pages=4, pages_per_sequence=4, left=-1, sinks=0)
    plan = dict(batch=1, heads=1, n_q=64, n_k=64, head_dim=64, dtype="bf16", cluster_q=16, cluster_k=16, keep=1, flags=0)
    for make, good in ((binding.make_window_problem, window), (binding.make_cache_problem, cache), (binding.make_problem, plan)):
        make(**good)
        for name in good:
            if name != "dtype":
                with pytest.raises(binding.ClusterAttnError):
                    make(**{**good, name: big})
    none = object.__new__(binding.PagedCache)
    none.problem = binding.make_cache_problem(**cache)
    with pytest.raises(binding.ClusterAttnError, match="appended"):
        none.paged_attention_fwd(None, appended=big)


def test_positions_without_rotary_are_refused():
    """They would be left aside without a word."""
    plan = object.__new__(binding.Plan)
    for args in (dict(positions_q=1), dict(positions_k=1)):
        with pytest.raises(binding.ClusterAttnError, match="positions without rotary"):
            plan.forward(None, None, None, **args)
        with pytest.raises(binding.ClusterAttnError, match="positions without rotary"):
            plan.forward_adaptive(None, None, None, 0.5, **args)


def test_an_output_that_is_the_queries_keeps_their_strides():
    build.build()
    lib = binding.load_library()
    cache = binding.make_cache_problem(batch=2, heads_q=8, heads_kv=2, head_dim=128, dtype="bf16", page_rows=16, pages=100, pages_per_sequence=20)
    at = 1 << 20                                            # (an address that nothing reads: the calls are refused)
    q = binding.CaRows(at, 1 << 16, 1 << 12, 128)
    for other in (binding.CaRows(at, 1 << 17, 1 << 12, 128), binding.CaRows(at, 1 << 16, 1 << 11, 128)):
        assert lib.paged_attention_fwd(cache, q, at, at, at, 0, at, other, None, at, 1 << 30, None) == 1
