"""The attention tests once more, by the chunk kernel also over the short caches that the single-token kernel would take."""
import types

import pytest
import torch

from paged_wide import widen
from test_paged_cache import (  # noqa: F401
    Case, test_attention_check_reports_a_wait_that_ran_out, test_attention_does_not_change_between_calls_streams_and_graphs,
    test_attention_extreme_scores, test_attention_head_layouts, test_attention_into_a_given_tensor, test_attention_long_cache_in_parts,
    test_attention_masks_and_scores, test_attention_max_new_is_a_hint, test_attention_of_many_requests_with_chunks,
    test_attention_offsets_past_32_bits, test_attention_pages_and_strides, test_attention_rows_without_keys, test_attention_scale,
    test_attention_table_entries_outside_the_cache_read_as_zeros, test_attention_types_and_lengths,
    test_attention_values_that_are_not_finite_reach_only_who_sees_them)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gorio():
    """The package, its attention with tables made wide."""
    from paper_2607_04415_b200 import build
    build.build()
    import paper_2607_04415_b200 as g
    held = []

    def paged_attention(q, key_pages, value_pages, tables, *args, **more):
        held.append(widen(tables, key_pages.shape[2]))
        if more.get("stream") is not None:
            torch.cuda.synchronize()
        return g.paged_attention(q, key_pages, value_pages, held[-1], *args, **more)
    return types.SimpleNamespace(paged_attention=paged_attention, attention_workspace=g.attention_workspace, attention_check=g.attention_check,
                                 cache_store=g.cache_store, GorioError=g.GorioError)


def test_wide_tables_choose_the_other_kernel(gorio):
    """The two kernels add in different orders: some last bits differ."""
    import paper_2607_04415_b200 as g
    c = Case([60, 40], [300, 200], dim=128)
    assert not torch.equal(c.check(g)["lse"], c.check(gorio)["lse"])
