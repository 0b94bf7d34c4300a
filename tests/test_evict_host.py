"""Eviction's refusals and the largest budgets, as far as no GPU is needed."""
import pytest

from tests.test_chunk_host import SHAPE, call, config, lib  # noqa: F401

LARGEST = 2147483647


@pytest.mark.parametrize("budget,batch", [(LARGEST, 4), (1 << 30, 8), ((1 << 30) + 1, 8)])
def test_more_pages_of_results_than_are_counted_are_refused_before_any_launch(lib, budget, batch):  # noqa: F811
    """(without a GPU a launch fails, with another status)"""
    assert call(lib, "ffd_evict_kv", budget=budget, batch=batch) == SHAPE
    assert call(lib, "ffd_evict_kv", budget=budget, batch=batch, n_sink=5, n_local=6) == SHAPE


def test_fewer_are_not(lib):  # noqa: F811
    for budget in (1, 64, LARGEST - 64, LARGEST - 63, LARGEST):
        # what is refused next is behind it: a workspace that is too small
        assert call(lib, "ffd_evict_kv", cfg=config(num_q_heads=4, num_kv_heads=1), batch=1, budget=budget, n_sink=0,
                    n_local=1, workspace_bytes=255) == 5
