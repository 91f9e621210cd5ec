"""The paged attention has no backward pass, and says so instead of cutting gradients off without a word."""
import pytest
import torch


@pytest.fixture(scope="module")
def gorio():
    from paper_2607_04415_b200 import build
    build.build()
    import paper_2607_04415_b200 as g
    return g


def test_results_refuse_gradients_where_an_input_asks_for_one(gorio):
    from paper_2607_04415_b200 import paged
    out, lse = torch.ones(4, 2), torch.ones(4)
    plain, asks = torch.zeros(3), torch.zeros(3, requires_grad=True)
    assert paged._without_gradient(out, None, (plain, plain, plain, None)) == (out, None)
    with torch.no_grad():
        assert paged._without_gradient(out, lse, (asks, plain, plain, None))[0] is out
    for inputs in ((asks, plain, plain, None), (plain, plain, plain, asks)):
        for with_lse in (lse, None):
            o, m = paged._without_gradient(out, with_lse, inputs)
            assert o.data_ptr() == out.data_ptr() and torch.equal(o.detach(), out) and (m is None) == (with_lse is None)
            for x in (o,) if m is None else (o, m):
                with pytest.raises(gorio.GorioError) as e:
                    x.sum().backward()
                assert e.value.status == 1 and "backward" in str(e.value)
    assert asks.grad is None


@pytest.mark.gpu
@pytest.mark.parametrize("new", [1, 140])
def test_attention_of_queries_that_ask_for_a_gradient(gorio, new):
    from test_paged_cache import Case
    c = Case([new], [300], dim=64)
    want = c.run(gorio)
    assert not want["out"].requires_grad
    c.q.requires_grad_()
    with torch.no_grad():
        got = c.run(gorio)
        assert torch.equal(got["out"], want["out"]) and not got["out"].requires_grad
    wide = torch.zeros_like(want["out"])
    got = c.run(gorio, out=wide)
    assert torch.equal(got["out"].detach(), want["out"]) and got["out"].data_ptr() == wide.data_ptr()
    for k in ("out", "lse"):
        with pytest.raises(gorio.GorioError):
            got[k].sum().backward()
    assert c.q.grad is None
