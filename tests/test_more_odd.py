"""Shared prefixes and quantised caches in the calls that are allowed and rare: results in other tensors' rows, scales at any address, caches without
pages, calls side by side, waits that run out."""
import pytest
import torch

from more_plain import assert_near
from test_prefix import Shared
from test_quantized import E4M3, INT8, Coded

pytestmark = pytest.mark.gpu

BF16, FP16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def gorio():
    from paper_2607_04415_b200 import build
    build.build()
    import paper_2607_04415_b200 as g
    yield g
    g.attention_wait_limit()


@pytest.mark.parametrize("new", [1, 130])
def test_results_go_to_rows_of_other_tensors(gorio, new):
    for c in (Shared([(300, [(new, new + 9)] * 3), (5, [(1, 4)])], dim=96), Coded([new, 1], [700, 90], dim=96), Coded([new, 1], [700, 90], dim=64, form=INT8)):
        t, heads, dim = c.q.shape
        wide = torch.full((t, heads + 2, dim + 16), 7.0, dtype=BF16, device="cuda")
        got = c.run(gorio, out=wide[:, 1:1 + heads, 8:8 + dim])
        assert_near(got, c.want())
        assert got["out"].data_ptr() == wide[:, 1:, 8:].data_ptr()
        wide[:, 1:1 + heads, 8:8 + dim] = 7.0
        assert (wide == 7.0).all()


@pytest.mark.parametrize("new", [1, 40, 200])
@pytest.mark.parametrize("off", [1, 3, 4])
def test_scales_at_any_address(gorio, new, off):
    """Scales that do not stand on 16 bytes, and such with odd rows between pages."""
    c = Coded([new, 3], [900, 200], dim=128, page=16)
    want = c.want()
    for name in ("ks", "vs"):
        s = getattr(c, name)
        flat = torch.zeros(s.numel() + 8, device="cuda")
        flat[off:off + s.numel()] = s.reshape(-1)
        setattr(c, name, flat[off:off + s.numel()].view(s.shape))
    assert_near(c.run(gorio), want)
    for name in ("ks", "vs"):
        s = getattr(c, name)
        wide = torch.zeros((s.shape[0], s.shape[1], s.shape[2] + off), device="cuda")
        wide[..., :s.shape[2]] = s
        setattr(c, name, wide[..., :s.shape[2]])
    assert_near(c.run(gorio), want)


@pytest.mark.parametrize("new", [1, 100])
def test_prefix_over_a_cache_without_pages(gorio, new):
    c = Shared([(100, [(new, new + 5)] * 3)])
    none = c.kp[:0]
    got = gorio.prefix_attention(c.q, none, none, c.prefix_tables, c.prefix_lengths, c.group_starts, c.tables, c.lengths, c.starts, new, want_lse=True, causal=False)
    assert (got["out"] == 0).all()
    keys = torch.tensor(float(100 + new + 5)).log()
    assert ((got["lse"].cpu() - keys).abs() <= 2.0 ** -18 + 2.0 ** -20 * keys).all()         # even weights of zeros


def test_calls_side_by_side(gorio):
    """Every operator on two streams at once, none waiting for the other."""
    cases = [(Shared([(3000, [(1, 50)] * 20)], dim=128, heads=8, kv_heads=2, seed=s), Coded([1] * 9 + [150], [3000] * 10, dim=128, seed=s)) for s in (1, 2)]
    want = [[x.run(gorio) for x in pair] for pair in cases]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for _ in range(15):
        for i, s in enumerate(streams):
            got[i].append([x.run(gorio, stream=s) for x in cases[i]])
    torch.cuda.synchronize()
    for i in range(2):
        for pair in got[i]:
            for a, b in zip(pair, want[i]):
                assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])


def after_limit(gorio, c, ws, limit, want):
    """A call under that limit, and one under none where a wait ran out."""
    gorio.attention_wait_limit(limit)
    got = c.run(gorio, workspace=ws)
    gorio.attention_wait_limit()
    try:
        gorio.attention_check(ws)
    except gorio.GorioError as e:
        assert e.status == 5 and "limit" in str(e)
        got = c.run(gorio, workspace=ws)
        gorio.attention_check(ws)
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"]) and (ws[: 1 << 16] == 0).all()


@pytest.mark.parametrize("which", ["two row tiles", "one row tile", "many units", "scored", "prefix", "prefix and chunks", "prefix of many units"])
def test_under_limits_that_some_waits_pass(gorio, which):
    """Waits may run out at any place, with copies and products under way: the call ends, says so, and the next one is right."""
    c = {"two row tiles": lambda: Coded([60], [9000], heads=8, kv_heads=1, dim=128),
         "one row tile": lambda: Coded([20], [9000], heads=4, kv_heads=1, dim=128, form=INT8),
         "many units": lambda: Coded([300] * 9, [700] * 9, heads=16, kv_heads=8, dim=96),
         "scored": lambda: Coded([100, 1, 700], [3000, 90, 900], heads=8, kv_heads=2, dim=64, dtype=FP16, softcap=30.0, slopes=True, window=500),
         "prefix": lambda: Shared([(9000, [(1, 30)] * 40)], heads=8, kv_heads=1, dim=128),
         "prefix and chunks": lambda: Shared([(3000, [(90, 400)] * 3), (40, [(1, 9)])], heads=8, kv_heads=2, dim=64, slopes=True),
         "prefix of many units": lambda: Shared([(700, [(300, 400)] * 2)] * 5, heads=16, kv_heads=8, dim=96)}[which]()
    ws = gorio.attention_workspace()
    want = c.run(gorio, workspace=ws)
    assert_near(want, c.want())
    gorio.attention_check(ws)
    for limit in (1e-9, 1.1e-6, 2.1e-6, 5e-6, 1e-5, 3e-5):
        for _ in range(3):
            after_limit(gorio, c, ws, limit, want)
