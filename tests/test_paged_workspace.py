"""Whose workspace an attention call uses, and what the checks of one refuse."""
import types

import pytest
import torch


@pytest.fixture(scope="module")
def gorio():
    from paper_2607_04415_b200 import build
    build.build()
    import paper_2607_04415_b200 as g
    return g


def test_a_captured_call_never_takes_the_streams_workspace(gorio, monkeypatch):
    from paper_2607_04415_b200 import paged
    made, state = [], types.SimpleNamespace(capturing=False)
    monkeypatch.setattr(paged, "attention_workspace", lambda device=None: made.append(object()) or made[-1])
    monkeypatch.setattr(paged, "_raw_stream", lambda index: 77)
    monkeypatch.setattr(paged, "_WORKSPACES", {})
    monkeypatch.setattr(paged, "_current_device", lambda: 0)
    monkeypatch.setattr(paged, "_current_stream_captured", lambda: state.capturing)
    kept = paged._stream_workspace(0)
    assert paged._stream_workspace(0) is kept
    state.capturing = True
    first, second = paged._stream_workspace(0), paged._stream_workspace(0)
    assert len({id(kept), id(first), id(second)}) == 3
    state.capturing = False
    assert paged._stream_workspace(0) is kept and len(made) == 3


@pytest.mark.gpu
@pytest.mark.parametrize("new", [30, 130])
def test_a_graph_beside_calls_on_the_stream_it_was_captured_on(gorio, new):
    from test_paged_cache import Case
    from paper_2607_04415_b200 import paged
    c = Case([1, new, 1], [5000, 900, 77], dim=128, heads=8, kv_heads=2)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    first = c.run(gorio, stream=s)                            # a warm-up: the stream has a workspace now
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        held = c.run(gorio)
    kept = paged._WORKSPACES[0, s.cuda_stream]
    kept[: (1 << 16) - 4] = 1                                 # as if a call on s were halfway
    before = kept.clone()
    held["out"].zero_()
    graph.replay()
    torch.cuda.synchronize()
    same, untouched = torch.equal(first["out"], held["out"]), torch.equal(kept, before)
    kept[: 1 << 16] = 0
    assert same and untouched


@pytest.mark.gpu
def test_calls_on_two_streams_overlap(gorio):
    """Twenty calls on each of two streams and replays of a graph on a third, none waiting for the others."""
    from test_paged_cache import Case
    cases = [Case([1, 1], [9000, 3000], dim=128, heads=8, kv_heads=2), Case([130, 40], [4000, 900], dim=64, heads=8, kv_heads=2)]
    want = [c.run(gorio) for c in cases]
    streams = [torch.cuda.Stream() for _ in range(3)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=streams[0]):
        held = [c.run(gorio) for c in cases]
    torch.cuda.synchronize()
    got = []
    for i in range(20):
        got += [(k, cases[k].run(gorio, stream=streams[k])) for k in range(2)]
        with torch.cuda.stream(streams[2]):
            graph.replay()
    torch.cuda.synchronize()
    for k, g in got + list(enumerate(held)):
        assert torch.equal(g["out"], want[k]["out"]) and torch.equal(g["lse"], want[k]["lse"])


def test_check_refuses_what_is_no_workspace(gorio):
    for bad in (torch.zeros(1 << 20, dtype=torch.uint8), [0] * 10, 7):
        with pytest.raises(gorio.GorioError) as e:
            gorio.attention_check(bad)
        assert e.value.status == 1 and "workspace" in str(e.value)


@pytest.mark.gpu
def test_check_refuses_tensors_that_are_no_workspace(gorio):
    """It reads a word 64 KB from the start and, where that is not 0, clears them: of a smaller tensor, its neighbours' memory."""
    good = gorio.attention_workspace()
    for bad in (good[:100], good[: 1 << 16], good.view(torch.int32), good[::2], torch.zeros((2, 2), device="cuda")):
        with pytest.raises(gorio.GorioError) as e:
            gorio.attention_check(bad)
        assert e.value.status == 1
    gorio.attention_check(good)


def test_streams_of_another_device_are_refused(gorio, monkeypatch):
    """The calls would run on the current stream of the tensors' device instead, ordered after nothing that `stream` holds."""
    from paper_2607_04415_b200 import paged

    class Stream:                                             # of cuda:1
        device_index = 1
    entered = []
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: entered.append(s))
    monkeypatch.setattr(paged, "_cuda_index", lambda name, t: 0)
    i, x = torch.zeros(2, dtype=torch.int32), torch.zeros(1)
    for call in (lambda s: gorio.page_tables(i, i, i, i, i, 16, 0, stream=s), lambda s: gorio.cache_store(x, x, x, x, x, stream=s),
                 lambda s: gorio.paged_attention(x, x, x, i, i, i, 1, stream=s), lambda s: gorio.attention_check(x, stream=s)):
        for stream in (Stream(), 12345):
            with pytest.raises(gorio.GorioError) as e:
                call(stream)
            assert e.value.status == 1 and "stream" in str(e.value)
    assert not entered
