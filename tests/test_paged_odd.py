"""Values that are not finite in tiles which some rows of a unit see and others do not: they reach the rows that see them, and those alone,
at the cost of the tile and not of the cache."""
import math

import pytest
import torch

from paged_wide import widen
from test_paged_cache import BF16, FP16, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gorio():
    from paper_2607_04415_b200 import build
    build.build()
    import paper_2607_04415_b200 as g
    yield g
    g.attention_wait_limit()


def place(c, r, key, column, value):
    page = c.kp.shape[2]
    c.vp[c.tables[r, key // page].item(), :, key % page, column] = value


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("dim", [64, 96, 128])
@pytest.mark.parametrize("new,lens,heads,kv_heads", [
    ([300], [700], 8, 8),                                     # a unit of 256 rows and one of 44, cut
    ([256, 128], [900, 1500], 2, 2),                          # one unit a request, one of 256 and one of 128 rows, cut
    ([300] * 12, [400] * 12, 16, 16),                         # more units than blocks: whole ones
    ([40] * 30, [500] * 30, 8, 8),                            # whole units of one row tile, several key tiles each
])
@pytest.mark.parametrize("opts", [{}, dict(window=150), dict(softcap=20.0), dict(causal=False, window=90)])
def test_values_that_are_not_finite_reach_who_sees_them(gorio, dtype, dim, new, lens, heads, kv_heads, opts):
    c = Case(new, lens, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, sharp=1.0, seed=dim, **opts)
    for r, (n, keys) in enumerate(zip(new, lens)):
        # at both edges of what the rows see: keys that the middle of the request's tokens sees last, and first through a window
        at = keys - n // 2
        place(c, r, at, 3, (math.inf, -math.inf, math.nan)[r % 3])
        place(c, r, at, dim - 1, math.inf)
        place(c, r, min(keys - 1, at + 9), dim - 1, -math.inf)
        if c.opts["window"]:
            place(c, r, max(0, keys - n // 2 - c.opts["window"]), 7, math.inf)
    got = c.check(gorio, max_new=1)
    c.tables = widen(c.tables, 16)
    chunk = c.check(gorio)
    assert torch.isfinite(chunk["lse"]).all() and not torch.isfinite(chunk["out"]).all()
    assert torch.equal(torch.isfinite(got["out"]), torch.isfinite(chunk["out"]))


def test_one_such_value_does_not_hold_up_a_long_call(gorio):
    """Twenty requests of 256 tokens over 20000 keys each: 0.4 ms, far from the fifth of a second that a wait may take here."""
    b, keys, n, kv = 20, 20000, 256, 8
    pages = b * (keys // 16)
    kp = torch.empty((pages, kv, 16, 64), dtype=BF16, device="cuda").normal_()
    vp = torch.empty_like(kp).normal_()
    tables = torch.arange(pages, dtype=torch.int32, device="cuda").view(b, -1)
    vp[tables[:, (keys - 2) // 16].long(), :, (keys - 2) % 16, 3] = math.inf
    q = torch.randn((b * n, kv, 64), device="cuda").to(BF16)
    lengths = torch.full((b,), keys, dtype=torch.int32, device="cuda")
    starts = torch.arange(b + 1, dtype=torch.int32, device="cuda") * n
    ws = gorio.attention_workspace()
    gorio.attention_wait_limit(0.2)
    out = gorio.paged_attention(q, kp, vp, tables, lengths, starts, n, workspace=ws)["out"].view(b, n, kv, 64)
    gorio.attention_check(ws)
    assert torch.isfinite(out[:, :-2]).all() and torch.isfinite(out[..., 4:]).all() and (out[:, -2:, :, 3] == math.inf).all()
