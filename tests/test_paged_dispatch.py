"""The choice between the two attention kernels: right on both sides of it, and never the one that is several times slower."""
import pytest
import torch

from test_paged_cache import BF16, FP16, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gorio():
    from paper_2607_04415_b200 import build
    build.build()
    import paper_2607_04415_b200 as g
    return g


@pytest.mark.parametrize("new,lens,heads,kv_heads,dim", [
    ([6], [150], 32, 8, 128), ([48], [150], 32, 8, 128), ([24], [3000], 32, 8, 128), ([9], [30000], 8, 2, 64), ([24], [30000], 8, 2, 96),
    ([24] * 8, [150] * 8, 8, 2, 64), ([1] * 20 + [100], [400] * 21, 8, 1, 128), ([7, 1, 0, 19], [12000, 40, 5, 700], 10, 2, 64)])
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_attention_of_few_rows_over_short_and_long_caches(gorio, new, lens, heads, kv_heads, dim, dtype):
    c = Case(new, lens, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, seed=sum(lens))
    c.check(gorio)
    c.check(gorio, max_new=1)                                 # the single-token kernel, whatever the sizes
    c.opts["window"] = 70
    c.check(gorio)


def test_a_short_question_reads_a_long_cache_once(gorio):
    """24 tokens over 131072 keys (537 MB): their keys take a single token's call some 90 us, and are not read anew for every four tokens,
    which would take five times as long."""
    keys, page = 131072, 64
    kp = torch.empty((keys // page, 8, page, 128), dtype=BF16, device="cuda").normal_()
    vp = torch.empty_like(kp).normal_()
    tables = torch.randperm(keys // page, device="cuda").int()[None]
    lengths = torch.tensor([keys], dtype=torch.int32, device="cuda")

    def time(new):
        q = torch.randn((new, 32, 128), device="cuda").to(BF16)
        starts = torch.tensor([0, new], dtype=torch.int32, device="cuda")
        best = []
        for i in range(12):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            for _ in range(5):
                gorio.paged_attention(q, kp, vp, tables, lengths, starts, new)
            b.record()
            b.synchronize()
            best.append(a.elapsed_time(b) / 5)
        return min(best[2:])
    one, short = time(1), time(24)
    assert short < 3 * one, f"24 tokens take {1e3 * short:.0f} us, one takes {1e3 * one:.0f} us"
