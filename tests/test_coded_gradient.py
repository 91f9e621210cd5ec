"""The calls on a quantised cache have no backward pass, and say so where an input asks for a gradient."""
import pytest
import torch

from test_quantized import E4M3, Coded


@pytest.fixture(scope="module")
def gorio():
    from paper_2607_04415_b200 import build
    build.build()
    import paper_2607_04415_b200 as g
    return g


def test_refusals_name_their_call(gorio):
    from paper_2607_04415_b200 import paged
    out, asks = torch.ones(4), torch.zeros(3, requires_grad=True)
    for more, call in (((), "paged_attention"), (("prefix_attention",), "prefix_attention"), (("cache_load_quantized",), "cache_load_quantized")):
        for x in paged._without_gradient(out, out.clone(), (asks, None), *more):
            with pytest.raises(gorio.GorioError) as e:
                x.sum().backward()
            assert str(e.value).split(": ", 1)[1].startswith(call + " has no backward pass")


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["ks", "vs", "kp", "vp"])
def test_caches_that_ask_for_a_gradient(gorio, name):
    c = Coded([1], [100], form=E4M3)
    slots = c.tables[0, :6].long() * c.page

    def load(**more):
        return gorio.cache_load_quantized(c.kp, c.vp, c.ks, c.vs, slots, **more)
    want, attended = load(), c.run(gorio)
    assert not want[0].requires_grad and not attended["out"].requires_grad
    getattr(c, name).requires_grad_()
    with torch.no_grad():
        assert not load()[0].requires_grad
    wide = torch.zeros((6, 8, 64), dtype=torch.bfloat16, device="cuda")
    for got in (load(), load(out=(wide[:, :4], wide[:, 4:]))):
        for x, y in zip(got, want):
            assert torch.equal(x.detach(), y)
            with pytest.raises(gorio.GorioError, match="cache_load_quantized"):
                x.float().sum().backward()
    assert torch.equal(wide[:, :4], want[0]) and torch.equal(wide[:, 4:], want[1])
    got = c.run(gorio)
    for k in ("out", "lse"):
        assert torch.equal(got[k].detach(), attended[k])
        with pytest.raises(gorio.GorioError, match="paged_attention_quantized"):
            got[k].float().sum().backward()
    assert getattr(c, name).grad is None
