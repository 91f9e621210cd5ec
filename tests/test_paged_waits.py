"""Waits inside the chunk kernel that run out: the call ends, attention_check says so, and the next call is right."""
import pytest
import torch

from paged_wide import widen
from test_paged_cache import BF16, FP16, Case


@pytest.fixture(scope="module")
def gorio():
    from paper_2607_04415_b200 import build
    build.build()
    import paper_2607_04415_b200 as g
    yield g
    g.attention_wait_limit()


def test_limits_that_are_none_are_refused(gorio):
    for bad in (-1.0, float("nan"), float("inf")):
        with pytest.raises(gorio.GorioError) as e:
            gorio.attention_wait_limit(bad)
        assert e.value.status == 1
    gorio.attention_wait_limit(10.0)


CASES = [
    ([130], [130], 8, 4, 64, BF16, {}),                                     # units of both sizes, few tiles
    ([60], [9000], 8, 1, 128, BF16, {}),                                    # two row tiles, cut between many blocks
    ([20], [9000], 4, 1, 128, FP16, {}),                                    # one row tile, its key tiles by turns
    ([300] * 9, [700] * 9, 16, 8, 96, BF16, {}),                            # more units than blocks
    ([100, 1, 700], [3000, 90, 900], 8, 2, 64, FP16, dict(softcap=30.0, slopes=True, window=500)),
]


def same(a, b):
    return all(torch.equal(a[k].nan_to_num(123.0), b[k].nan_to_num(123.0)) for k in ("out", "lse"))


def after_limit(gorio, c, ws, limit, want):
    """A call under that limit, and one under none where a wait ran out; whether one did."""
    gorio.attention_wait_limit(limit)
    got = c.run(gorio, workspace=ws)
    gorio.attention_wait_limit()
    ran_out = False
    try:
        gorio.attention_check(ws)
    except gorio.GorioError as e:
        assert e.status == 5 and "limit" in str(e)
        ran_out = True
        got = c.run(gorio, workspace=ws)
        gorio.attention_check(ws)
    assert same(got, want) and (ws[: 1 << 16] == 0).all()
    return ran_out


@pytest.mark.gpu
@pytest.mark.parametrize("new,lens,heads,kv_heads,dim,dtype,opts", CASES)
def test_attention_under_limits_that_some_waits_pass(gorio, new, lens, heads, kv_heads, dim, dtype, opts):
    """Waits may run out at any place, with copies and products under way."""
    c = Case(new, lens, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, **opts)
    c.tables = widen(c.tables, c.kp.shape[2])
    ws = gorio.attention_workspace()
    want = c.check(gorio, workspace=ws)
    gorio.attention_check(ws)
    for limit in (1e-9, 1.1e-6, 2.1e-6, 5e-6, 1e-5, 3e-5):
        for _ in range(3):
            after_limit(gorio, c, ws, limit, want)


@pytest.mark.gpu
@pytest.mark.parametrize("new,lens,heads,kv_heads,dim,dtype,opts", CASES[1:4] + [([250], [9000], 2, 2, 128, BF16, {})])
def test_attention_whose_waits_run_out_says_so(gorio, new, lens, heads, kv_heads, dim, dtype, opts):
    """A value that is not finite and that some rows do not see: the warps whose rows read the cache for it keep others waiting for far
    longer than the limit."""
    c = Case(new, lens, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, **opts)
    for r, n in enumerate(lens):
        c.vp[c.tables[r, (n - 2) // 16].item(), :, (n - 2) % 16, 3] = float("inf")
    c.tables = widen(c.tables, c.kp.shape[2])
    ws = gorio.attention_workspace()
    want = c.run(gorio, workspace=ws)
    gorio.attention_check(ws)
    for limit in (1e-9, 1.1e-6, 5e-6):
        assert after_limit(gorio, c, ws, limit, want)
