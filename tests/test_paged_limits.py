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


@pytest.mark.gpu
@pytest.mark.parametrize("new", [1, 200])
@pytest.mark.parametrize("dim,page", [(64, 16), (96, 8), (128, 64)])
def test_attention_over_a_cache_without_pages(gorio, new, dim, page):
    """All table entries lie outside it, so that every key reads as zeros: even weights of values that are 0."""
    pages = torch.empty((0, 2, page, dim), dtype=torch.bfloat16, device="cuda")
    q = torch.randn((new, 4, dim), device="cuda").bfloat16()
    tables = torch.full((1, 300 // page + 1), -1, dtype=torch.int32, device="cuda")
    lengths, starts = torch.tensor([300], dtype=torch.int32, device="cuda"), torch.tensor([0, new], dtype=torch.int32, device="cuda")
    got = gorio.paged_attention(q, pages, pages, tables, lengths, starts, new, want_lse=True)
    sees = torch.arange(301 - new, 301, device="cuda").float()
    assert (got["out"] == 0).all()
    assert ((got["lse"] - sees.log()[:, None]).abs() <= 2.0 ** -18 + 2.0 ** -20 * sees.log()[:, None]).all()
    gorio.cache_store(q[:, :2], q[:, 2:], pages, pages, torch.zeros(new, dtype=torch.int64, device="cuda"))
    torch.cuda.synchronize()
