"""Attention of batches whose requests share prefixes, against one softmax in 64 bits over the prefix and each request's own keys."""
import math
import random

import pytest
import torch

from more_plain import assert_near, attend
from paged_plain import ceil_div

pytestmark = pytest.mark.gpu

BF16, FP16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def gorio():
    from paper_2607_04415_b200 import build
    build.build()
    import paper_2607_04415_b200 as g
    return g


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Shared:
    """Groups [(prefix tokens, [(new tokens, own keys), ...]), ...]; `before` and `after` are requests of no group.  Whatever no query sees
    is NaN."""

    def __init__(self, groups, heads=8, kv_heads=4, dim=64, page=16, dtype=BF16, seed=0, layout="heads", causal=True, window=0, softcap=0.0, slopes=False,
                 before=(), after=(), spare=0, sharp=2.0, freed=False):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.members = list(before) + [m for _, ms in groups for m in ms] + list(after)
        self.ahead = [0] * len(before) + [p for p, ms in groups for _ in ms] + [0] * len(after)
        self.group_of = [None] * len(before) + [i for i, (_, ms) in enumerate(groups) for _ in ms] + [None] * len(after)
        self.prefixes = [p for p, _ in groups]
        lens, self.new = [k for _, k in self.members], [n for n, _ in self.members]
        held = sum(ceil_div(n, page) for n in lens + self.prefixes)
        shape = (held + 4 + spare, kv_heads, page, dim)

        def cache():
            if layout == "tokens":
                return torch.full((shape[0], page, kv_heads, dim), math.nan, dtype=dtype, device="cuda").transpose(1, 2)
            return torch.full(shape, math.nan, dtype=dtype, device="cuda")
        self.kp, self.vp = cache(), cache()
        order = (torch.randperm(held + 4, generator=g, device="cuda") + spare).tolist()

        def fill(all_lens, gone):
            width = max([1] + [ceil_div(n, page) for n in all_lens]) + 1
            tables = [[-1] * width for _ in all_lens]
            for r, n in enumerate(all_lens):
                for i in range(ceil_div(n, page)):
                    tables[r][i] = order.pop()
                    rows = min(page, n - i * page)
                    self.kp[tables[r][i], :, :rows] = torch.randn((kv_heads, rows, dim), generator=g, device="cuda").to(dtype)
                    self.vp[tables[r][i], :, :rows] = torch.randn((kv_heads, rows, dim), generator=g, device="cuda").to(dtype)
                for i in range(gone(r)):                           # pages that lie before every query's window are given back
                    tables[r][i] = -1 if (i + r) % 2 else (1 << 30)
            return _i32(tables).view(len(all_lens), width)
        self.tables = fill(lens, lambda r: 0)
        first = [min([p + k - n for n, k in ms] + [p]) for p, ms in groups]
        self.prefix_tables = fill(self.prefixes, lambda i: max(0, first[i] - window + 1) // page if freed else 0)
        self.lens, self.page = lens, page
        self.lengths, self.prefix_lengths = _i32(lens), _i32(self.prefixes)
        self.starts = _i32([sum(self.new[:i]) for i in range(len(self.new) + 1)])
        self.group_starts = _i32([len(before) + sum(len(ms) for _, ms in groups[:i]) for i in range(len(groups) + 1)])
        self.q = torch.randn((sum(self.new), heads, dim), generator=g, device="cuda").mul_(sharp).to(dtype)
        self.opts = dict(causal=causal, window=window, softcap=softcap,
                         slopes=torch.exp2(-torch.arange(1, heads + 1, device="cuda") / 2).float() if slopes else None)

    def run(self, gorio, **more):
        return gorio.prefix_attention(self.q, self.kp, self.vp, self.prefix_tables, self.prefix_lengths, self.group_starts, self.tables, self.lengths,
                                      self.starts, more.pop("max_new", max([1] + self.new)), want_lse=True, **{**self.opts, **more})

    def _rows(self, pages, ids, n):
        ids = torch.where((ids < 0) | (ids >= pages.shape[0]), 0, ids).long()
        return pages[ids].transpose(0, 1).reshape(pages.shape[1], -1, pages.shape[3])[:, :n].double()

    def want(self):
        parts = []
        for r, (n, own) in enumerate(self.members):
            p, g = self.ahead[r], self.group_of[r]
            k, v = [torch.cat(([self._rows(x, self.prefix_tables[g, :ceil_div(p, self.page)], p)] if p else [])
                              + [self._rows(x, self.tables[r, :ceil_div(own, self.page)], own)], 1) for x in (self.kp, self.vp)]
            at = torch.arange(p + own - n, p + own, device="cuda")
            j = torch.arange(p + own, device="cuda")
            sees = torch.ones((n, p + own), dtype=torch.bool, device="cuda")
            if self.opts["causal"]:
                sees &= (j[None] <= at[:, None]) | (j[None] < p)
            if self.opts["window"]:
                sees &= j[None] > at[:, None] - self.opts["window"]
            parts.append(attend(self.q[self.starts[r]:self.starts[r + 1]], k, v, sees, j[None] - at[:, None], self.opts["softcap"], self.opts["slopes"]))
        return [torch.cat(x) for x in zip(*parts)]

    def check(self, gorio, **more):
        got = self.run(gorio, **more)
        assert_near(got, self.want())
        return got


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("dim", [64, 96, 128])
@pytest.mark.parametrize("groups", [[(1, [(1, 1)])], [(100, [(1, 1), (1, 30), (1, 200)])], [(130, [(1, 5)] * 40)], [(777, [(3, 50), (40, 40), (1, 0), (2, 700)])],
                                    [(40, [(1, 2), (5, 5)]), (0, [(1, 9)]), (600, [(1, 1)] * 17), (9, []), (33, [(70, 90)])]])
def test_prefix_types_and_lengths(gorio, dtype, dim, groups):
    Shared(groups, dim=dim, dtype=dtype, seed=dim).check(gorio)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 1), (3, 3), (14, 2), (32, 2)])
@pytest.mark.parametrize("members", [[(1, 7)], [(1, 30), (1, 1), (1, 100)], [(1, i) for i in range(70)], [(200, 200), (1, 3)]])
def test_prefix_head_layouts(gorio, heads, kv_heads, members):
    Shared([(300, members), (20, members[:1])], heads=heads, kv_heads=kv_heads, dim=128, seed=heads).check(gorio)


@pytest.mark.parametrize("page", [8, 16, 24, 64, 256])
@pytest.mark.parametrize("layout", ["heads", "tokens"])
@pytest.mark.parametrize("length", [1, 15, 16, 17, 511, 1024])
def test_prefix_pages_that_end_anywhere(gorio, page, layout, length):
    Shared([(length, [(1, 40)] * 3), (length + 1, [(33, 60)] * 2)], page=page, layout=layout, seed=page).check(gorio)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [0, 1, 20, 90, 400])
@pytest.mark.parametrize("softcap,slopes", [(0.0, False), (5.0, False), (0.0, True), (100.0, True)])
@pytest.mark.parametrize("new", [1, 30])
def test_prefix_masks_and_scores(gorio, causal, window, softcap, slopes, new):
    groups = [(300, [(new, new), (1, 120), (new, new + 33), (1, 0)]), (150, [(new, new)] * 9), (70, [(1, 300)])]
    Shared(groups, dim=128 if softcap else 64, causal=causal, window=window, softcap=softcap, slopes=slopes, seed=window, freed=window > 0).check(gorio)


@pytest.mark.parametrize("causal", [True, False])
def test_prefix_rows_without_keys(gorio, causal):
    got = Shared([(0, [(1, 0), (3, 0)]), (5, [(2, 0)])], causal=causal, before=[(2, 0), (1, 20)], after=[(4, 10), (30, 0)]).check(gorio)
    assert (got["out"][:2] == 0).all() and (got["lse"][:2] == -math.inf).all() and (got["lse"][-30:] == -math.inf).all()
    Shared([(64, [])], before=[(1, 30)], after=[(0, 4), (3, 5)], causal=causal).check(gorio)
    Shared([(64, [(0, 9)]), (30, [(0, 0), (1, 1)])], causal=causal).check(gorio)
    Shared([(400, [(1, 0)] * 50)], causal=causal).check(gorio)                            # nothing but the prefix
    Shared([(400, [(60, 10), (3, 0)])], causal=causal, slopes=True).check(gorio)          # fewer own keys than new tokens
    c = Shared([(64, [(0, 3)])], causal=causal)
    assert c.run(gorio)["out"].shape == (0, 8, 64)


def test_prefix_of_many_requests_and_groups(gorio):
    rng = random.Random(3)
    Shared([(rng.randint(0, 90), [(rng.randint(0, 2), rng.randint(0, 40)) for _ in range(rng.randint(0, 6))]) for _ in range(300)], heads=2, kv_heads=1).check(gorio)
    Shared([(5000, [(1, rng.randint(0, 40)) for _ in range(700)])], heads=2, kv_heads=1, slopes=True).check(gorio)


@pytest.mark.parametrize("members", [[(1, 9)], [(1, 30)] * 33])
def test_prefix_long(gorio, members):
    Shared([(40000, members)], heads=8, kv_heads=2, dim=128, page=64).check(gorio)
    Shared([(20000, members), (7000, members * 2)], heads=8, kv_heads=1, page=64, window=9000).check(gorio)


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_prefix_values_that_are_not_finite_reach_only_who_sees_them(gorio, new, bad):
    # under a window of 50 only the first request's first tokens see key 270 of 300
    c = Shared([(300, [(new, new), (new, 100 + new)])], window=50, heads=8, kv_heads=2)
    c.vp[c.prefix_tables[0, 270 // 16].item(), :, 270 % 16, 3] = bad
    got = c.check(gorio)
    assert not torch.isfinite(got["out"][0, :, 3]).any() and torch.isfinite(got["out"][0, :, 4]).all() and torch.isfinite(got["out"][new:]).all()
    c = Shared([(300, [(new, new)] * 3)], heads=8, kv_heads=2)
    c.kp[c.prefix_tables[0, 3].item(), :, 3, 3] = math.nan
    assert torch.isnan(c.run(gorio)["out"]).all()


@pytest.mark.parametrize("members", [[(1, 30), (1, 77)], [(1, 40)] * 40, [(60, 200)] * 2])
def test_prefix_is_what_one_table_of_both_gives(gorio, members):
    """A prefix of whole pages may as well stand in each request's own table: the same numbers but for roundings, which both sides'
    tolerances count."""
    c = Shared([(320, members)], dim=128, heads=8, kv_heads=2, slopes=True)
    got = c.check(gorio)
    both = torch.cat([c.prefix_tables[:, :20].expand(len(members), -1), c.tables], 1).contiguous()
    one = gorio.paged_attention(c.q, c.kp, c.vp, both, c.lengths + 320, c.starts, members[0][0], want_lse=True, **c.opts)
    assert_near(one, c.want())
    assert (got["out"].double() - one["out"].double()).abs().max() < 0.05


def test_prefix_offsets_past_32_bits(gorio):
    spare = (1 << 31) // (2 * 64 * 128) + 8
    for members in ([(1, 100)], [(1, 100)] * 60):
        Shared([(500, members)], dim=128, heads=4, kv_heads=2, page=64, spare=spare).check(gorio)
        torch.cuda.empty_cache()


def test_prefix_bad_numbers_stay_in_bounds(gorio):
    """Lengths, starts and table entries of any value are cut; other groups' results do not change."""
    c = Shared([(100, [(1, 20), (2, 30)]), (200, [(1, 5), (1, 6)])])
    want = c.run(gorio)
    big = (1 << 31) - 1
    for lengths in ([100, -5], [100, big], [100, -big]):
        c.prefix_lengths.copy_(_i32(lengths))
        got = c.run(gorio)
        assert torch.equal(got["out"][:3], want["out"][:3])
    c.prefix_lengths.copy_(_i32([100, 200]))
    for at, starts in ((0, [-7, 2, 4]), (0, [0, 2, 9]), (0, [0, 2, big]), (3, [-big, big, big])):
        c.group_starts.copy_(_i32(starts))
        got = c.run(gorio)
        if at == 0:
            assert torch.equal(got["out"], want["out"])
    c.group_starts.copy_(_i32([0, 2, 4]))
    c.prefix_tables[1, :] = -1                                   # reads as zeros
    got = c.run(gorio)
    assert torch.equal(got["out"][:3], want["out"][:3]) and torch.isfinite(got["out"]).all()
    torch.cuda.synchronize()


def test_prefix_rows_behind_the_last_request_are_left_as_they_were(gorio):
    c = Shared([(100, [(1, 20), (2, 30)])])
    c.q = torch.cat([c.q, torch.full_like(c.q[:2], math.nan)])
    out = torch.full_like(c.q, 7.0)
    c.run(gorio, out=out)
    assert (out[3:] == 7.0).all()
    c.q, out = c.q[:3], out[:3]
    assert_near(dict(out=out, lse=c.run(gorio)["lse"]), c.want())


@pytest.mark.parametrize("members", [[(1, 50)], [(1, 50), (1, 900)] * 20, [(90, 300), (1, 4)]])
def test_prefix_in_graphs_and_on_streams(gorio, members):
    """Two captured calls, replayed beside each other and beside calls on the stream they were captured on; lengths that grow between replays."""
    c, d = [Shared([(1500, members), (40, members[:1])], seed=s, heads=8, kv_heads=2, dim=128) for s in (1, 2)]
    want = [x.run(gorio) for x in (c, d)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.run(gorio)
    torch.cuda.synchronize()
    graphs, got = [], []
    for x in (c, d):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            got.append(x.run(gorio))
        graphs.append(g)
    for _ in range(20):
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
            more = c.run(gorio)
        last = d.run(gorio)
    torch.cuda.synchronize()
    for x, y in ((got[0], want[0]), (got[1], want[1]), (more, want[0]), (last, want[1])):
        assert torch.equal(x["out"], y["out"]) and torch.equal(x["lse"], y["lse"])
    c.prefix_lengths.sub_(7)
    c.prefixes = [p - 7 for p in c.prefixes]
    c.ahead = [p - 7 for p in c.ahead]
    graphs[0].replay()
    torch.cuda.synchronize()
    assert_near(got[0], c.want())
    ws = gorio.attention_workspace()
    assert torch.equal(c.run(gorio, workspace=ws)["out"], got[0]["out"])
    gorio.attention_check(ws)
    gorio.attention_check()
    del graphs


def test_prefix_results_do_not_change_from_call_to_call(gorio):
    """Many calls back to back, each of which may begin before the one before has ended: none reads another's results."""
    cases = [Shared([(700 + 300 * s, [(1, 20 * s + 1)] * (3 + 9 * s))], seed=s, heads=8, kv_heads=2, dim=128) for s in range(3)]
    want = [x.run(gorio)["out"] for x in cases]
    torch.cuda.synchronize()
    got = [(i, cases[i].run(gorio)["out"]) for _ in range(40) for i in (0, 1, 2, 1)]
    for i, out in got:
        assert torch.equal(out, want[i])


def test_prefix_refusals(gorio):
    c = Shared([(100, [(1, 20), (2, 30)])])
    good = dict(q=c.q, key_pages=c.kp, value_pages=c.vp, prefix_tables=c.prefix_tables, prefix_lengths=c.prefix_lengths, group_starts=c.group_starts,
                tables=c.tables, lengths=c.lengths, starts=c.starts, max_new=2)
    for name, bad in (("q", c.q.half()), ("q", c.q[:, :3]), ("q", c.q[..., :32]), ("key_pages", c.kp.half()), ("prefix_tables", c.prefix_tables.long()),
                      ("prefix_tables", c.prefix_tables[:0]), ("prefix_lengths", c.prefix_lengths.long()), ("prefix_lengths", c.prefix_lengths[:0]),
                      ("group_starts", c.group_starts[:1]), ("group_starts", c.group_starts.cpu()), ("lengths", c.lengths[:1]), ("starts", c.starts[:1]),
                      ("tables", c.tables[:1]), ("max_new", -1)):
        with pytest.raises(gorio.GorioError) as e:
            gorio.prefix_attention(**{**good, name: bad})
        assert e.value.status == 1
    for more in (dict(scale=0.0), dict(softcap=-1.0), dict(window=-1), dict(workspace=torch.zeros(9, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(gorio.GorioError):
            gorio.prefix_attention(**good, **more)
    q = c.q.clone().requires_grad_()
    with pytest.raises(gorio.GorioError):
        gorio.prefix_attention(**{**good, "q": q})["out"].sum().backward()
