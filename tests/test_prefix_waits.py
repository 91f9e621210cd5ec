"""The limit of a wait inside the last prefix kernel does not count the time that the kernels before it take."""
import math

import pytest
import torch

from test_prefix import Shared

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gorio():
    from paper_2607_04415_b200 import build
    build.build()
    import paper_2607_04415_b200 as g
    yield g
    g.attention_wait_limit()


def test_a_long_first_kernel_is_no_wait_that_runs_out(gorio):
    """One value of the prefix is infinite, which under a window keeps the blocks of one key head far longer than the others: on those the last
    kernel has begun, several parts a block, and waits for the first one's end."""
    c = Shared([(65536, [(64, 64)] * 64)], heads=8, kv_heads=8, dim=64, page=64, window=1 << 20)
    ws = gorio.attention_workspace()

    def call():
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        torch.cuda.synchronize()
        a.record()
        got = c.run(gorio, workspace=ws)
        b.record()
        b.synchronize()
        return got, a.elapsed_time(b) * 1e-3
    call()
    plain, quick = call()
    c.vp[c.prefix_tables[0, 0].item(), 0, 5, 3] = math.inf
    want, slow = call()
    gorio.attention_check(ws)
    limit = slow / 4
    assert quick < limit / 2, f"the first kernel takes {1e3 * slow:.2f} ms, {1e3 * quick:.2f} without the infinity"
    gorio.attention_wait_limit(limit)
    got, _ = call()
    gorio.attention_check(ws)
    gorio.attention_wait_limit()
    assert all(torch.equal(got[k].nan_to_num(9.0), want[k].nan_to_num(9.0)) for k in ("out", "lse"))
    assert torch.equal(got["out"][:, 1:], plain["out"][:, 1:])
