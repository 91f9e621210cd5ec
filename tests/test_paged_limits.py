"""Sizes at the ends of what the paged-cache calls take."""
import pytest
import torch


@pytest.fixture(scope="module")
def gorio():
    from paper_2607_04415_b200 import build
    build.build()
    import paper_2607_04415_b200 as g
    return g


def test_store_refuses_more_tokens_than_its_kernel_counts(gorio):
    """Close to 2^32 tokens the number of blocks wrapped around and almost nothing was stored."""
    import paper_2607_04415_b200.paged as p
    lib, at = gorio.load_library(), 1 << 20                   # an address that is never read: the calls are refused
    for tokens in (1 << 31, (1 << 32) - 1):
        store = [at] * 5 + [8, 8, 8, 8, 128, 128, 8, 128, 128, 8] + [tokens, 1, 8, 9, 16, 0]
        assert lib.gorio_cache_store(p._STORE.pack(*store), None) == 1
        assert b"tokens" in lib.gorio_last_error(None)
