"""The paged key/value cache on the GPU: page tables against a loop over requests, the store against
indexing (both exact), attention against 64 bits within the error that its formulas allow."""
import math
import random

import pytest
import torch

from paged_plain import ceil_div, plain_attention, plain_tables

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


# ---------------------------------------------------------------- page tables

def _check_tables(gorio, lengths, new_lens, width, page, free_count=None, n_tokens=None, seed=0, slack=3, table_pad=0):
    rng = random.Random(seed)
    held = [ceil_div(max(c, 0), page) for c in lengths]
    need = sum(max(0, ceil_div(max(c, 0) + max(n, 0), page) - h) for c, n, h in zip(lengths, new_lens, held))
    ids = list(range(sum(held) + need + slack))
    rng.shuffle(ids)
    tables, at = [], 0
    for h in held:
        row = ids[at:at + h][:width]
        at += h
        tables.append(row + [-1] * (width - len(row)))
    free = ids[at:]
    fc = len(free) if free_count is None else free_count
    t = sum(max(n, 0) for n in new_lens) if n_tokens is None else n_tokens
    want = plain_tables(lengths, new_lens, tables, free, fc, page, t)
    wide = torch.full((len(lengths), width + table_pad), -7, dtype=torch.int32, device="cuda")
    if tables:
        wide[:, :width] = _i32(tables).view(len(tables), width)
    got = gorio.page_tables(_i32(lengths), _i32(new_lens), wide[:, :width], _i32(free), _i32([fc]), page, t)
    for k, v in want.items():
        assert got[k].tolist() == v, k
    assert (wide[:, width:] == -7).all()
    return got


@pytest.mark.parametrize("page", [1, 8, 16, 24, 128])
@pytest.mark.parametrize("requests,new,cached", [(1, 1, 0), (1, 1, 15), (1, 1, 16), (1, 4000, 777), (7, 1, 300), (33, 40, 0), (1023, 3, 50), (1025, 2, 9),
                                                 (3000, 5, 40)])
def test_page_tables_follow_the_rules(gorio, page, requests, new, cached):
    rng = random.Random(requests * 31 + page)
    lengths = [rng.randint(0, cached) for _ in range(requests)] if requests > 1 else [cached]
    new_lens = [rng.randint(0, new) for _ in range(requests)] if requests > 1 else [new]
    width = max(1, max(ceil_div(c + n, page) for c, n in zip(lengths, new_lens))) + 1
    _check_tables(gorio, lengths, new_lens, width, page, seed=page, table_pad=requests % 3)


def test_page_tables_of_nothing(gorio):
    _check_tables(gorio, [5, 0, 16], [0, 0, 0], 4, 16)
    _check_tables(gorio, [], [], 1, 16)
    _check_tables(gorio, [0], [1], 1, 16)


def test_page_tables_serve_in_order_until_pages_run_out(gorio):
    lengths, new_lens = [15, 0, 16, 3, 0, 40], [2, 33, 1, 2, 0, 9]      # needs 1, 3, 1, 0, 0, 1 pages of 16
    for fc in range(8):
        got = _check_tables(gorio, lengths, new_lens, 6, 16, free_count=fc)
        assert got["served"].tolist() == [1 if n <= fc else 0 for n in (1, 4, 5, 5, 5, 6)]
    assert _check_tables(gorio, lengths, new_lens, 6, 16, free_count=-3)["free_count"].tolist() == [0]
    _check_tables(gorio, lengths, new_lens, 6, 16, free_count=1000)    # more than the stack holds: cut to it


def test_page_tables_refuse_single_requests(gorio):
    # a row too short, negative numbers: those requests alone are not served
    got = _check_tables(gorio, [10, 60, -1, 4, 8], [1, 10, 3, -2, 2], 4, 16)
    assert got["served"].tolist() == [1, 0, 0, 0, 1]
    # more new tokens than the outputs have rows for, and fewer
    _check_tables(gorio, [10, 0, 5], [3, 9, 2], 4, 16, n_tokens=12)
    _check_tables(gorio, [10, 0, 5], [3, 9, 2], 4, 16, n_tokens=20)
    big = (1 << 31) - 1
    _check_tables(gorio, [0, 3], [2, 1], 4, 16, n_tokens=3)
    got = gorio.page_tables(_i32([5, big, 3]), _i32([big, 1, 1]), _i32([[0], [1], [2]]), _i32([9, 8]), _i32([2]), 16, 3)
    assert got["served"].tolist() == [0, 0, 0] and got["free_count"].tolist() == [2]


def test_page_tables_step_by_step_match_one_step(gorio):
    """Ten single-token steps end in the tables of one step of ten."""
    free = _i32(list(range(50, 0, -1)))
    tables = torch.full((3, 4), -1, dtype=torch.int32, device="cuda")
    lengths, count = _i32([0, 0, 0]), _i32([50])
    seen = []
    for _ in range(10):
        got = gorio.page_tables(lengths, _i32([1, 1, 1]), tables, free, count, 8, 3)
        lengths, count = got["lengths"], got["free_count"]
        seen.append(got["slots"].tolist())
    assert lengths.tolist() == [10, 10, 10] and count.tolist() == [44]
    assert [[s[r] % 8 for s in seen] for r in range(3)] == [[p % 8 for p in range(10)]] * 3
    assert [[s[r] // 8 for s in seen] for r in range(3)] == [[tables[r, p // 8].item() for p in range(10)] for r in range(3)]
    assert len(set(x for s in seen for x in s)) == 30


# ---------------------------------------------------------------- store

@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("tokens,heads,dim,page", [(1, 1, 64, 8), (1, 8, 128, 16), (63, 3, 96, 24), (1000, 2, 128, 16), (257, 5, 8, 1)])
@pytest.mark.parametrize("layout", ["heads", "tokens", "joint"])
def test_cache_store(gorio, dtype, tokens, heads, dim, page, layout):
    g = torch.Generator(device="cuda").manual_seed(tokens)
    pages = ceil_div(tokens, page) + 3
    kv = torch.randn((tokens, 2, heads, dim), generator=g, device="cuda").to(dtype)
    k, v = (kv[:, 0], kv[:, 1]) if layout == "joint" else (kv[:, 0].contiguous(), kv[:, 1].contiguous())

    def cache():
        if layout == "tokens":
            return torch.randn((pages, page, heads, dim), generator=g, device="cuda").to(dtype).transpose(1, 2)
        return torch.randn((pages, heads, page, dim), generator=g, device="cuda").to(dtype)
    kp, vp = cache(), cache()
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:tokens]
    if tokens > 5:
        slots[2::5] = -1
    want_k, want_v = kp.clone(), vp.clone()
    for t, s in enumerate(slots.tolist()):
        if s >= 0:
            want_k[s // page, :, s % page] = k[t]
            want_v[s // page, :, s % page] = v[t]
    gorio.cache_store(k, v, kp, vp, slots)
    assert torch.equal(kp, want_k) and torch.equal(vp, want_v)
    # slots outside the cache are skipped
    gorio.cache_store(k, v, kp, vp, torch.full((tokens,), pages * page, device="cuda"))
    gorio.cache_store(k[:0], v[:0], kp, vp, slots[:0])
    assert torch.equal(kp, want_k) and torch.equal(vp, want_v)


# ---------------------------------------------------------------- attention

class Case:
    """A cache with the given requests in scattered pages; whatever no query sees is NaN."""

    def __init__(self, new, lens, heads=8, kv_heads=4, dim=64, page=16, dtype=BF16, seed=0, layout="heads", causal=True, window=0, softcap=0.0,
                 slopes=False, spare=0, sharp=2.0, freed=False):
        g = torch.Generator(device="cuda").manual_seed(seed)
        width = max(1, max(ceil_div(n, page) for n in lens)) + 1
        held = sum(ceil_div(n, page) for n in lens)
        shape = (held + 4 + spare, kv_heads, page, dim)

        def cache():
            if layout == "tokens":
                return torch.full((shape[0], page, kv_heads, dim), math.nan, dtype=dtype, device="cuda").transpose(1, 2)
            if layout == "joint":
                return torch.full((shape[0], kv_heads, page, dim + 16), math.nan, dtype=dtype, device="cuda")[..., 8:8 + dim]
            return torch.full(shape, math.nan, dtype=dtype, device="cuda")
        self.kp, self.vp = cache(), cache()
        order = (torch.randperm(held + 4, generator=g, device="cuda") + spare).tolist()
        tables = [[-1] * width for _ in lens]
        self.lens, self.new = lens, new
        for r, n in enumerate(lens):
            for i in range(ceil_div(n, page)):
                tables[r][i] = order.pop()
                rows = min(page, n - i * page)
                self.kp[tables[r][i], :, :rows] = torch.randn((kv_heads, rows, dim), generator=g, device="cuda").to(dtype)
                self.vp[tables[r][i], :, :rows] = torch.randn((kv_heads, rows, dim), generator=g, device="cuda").to(dtype)
        if freed:                                              # pages that lie before every query's window are given back
            for r, n in enumerate(lens):
                for i in range(max(0, n - new[r] - window + 1) // page):
                    tables[r][i] = -1 if (i + r) % 2 else (1 << 30)
        self.tables, self.lengths = _i32(tables), _i32(lens)
        self.starts = _i32([sum(new[:i]) for i in range(len(new) + 1)])
        t = sum(new)
        q = torch.randn((t, heads, dim), generator=g, device="cuda").mul_(sharp).to(dtype)
        if layout == "joint":                                  # a projection's columns
            wide = torch.zeros((t, heads + 3, dim), dtype=dtype, device="cuda")
            wide[:, 1:1 + heads] = q
            q = wide[:, 1:1 + heads]
        self.q = q
        self.max_new = max(new) if new else 0
        self.opts = dict(causal=causal, window=window, softcap=softcap,
                         slopes=torch.exp2(-torch.arange(1, heads + 1, device="cuda") / 2).float() if slopes else None)

    def run(self, gorio, **more):
        return gorio.paged_attention(self.q, self.kp, self.vp, self.tables, self.lengths, self.starts, more.pop("max_new", self.max_new),
                                     want_lse=True, **{**self.opts, **more})

    def check(self, gorio, **more):
        got = self.run(gorio, **more)
        self.compare(got)
        return got

    def compare(self, got):
        out, lse, out_tol, lse_tol = plain_attention(self.q, self.kp, self.vp, self.tables, self.lengths, self.starts, **self.opts)
        d = got["out"].double() - out
        same = (got["out"].double() == out) | (torch.isnan(out) & torch.isnan(got["out"]))
        assert ((d.abs() <= out_tol) | same).all(), f"off by {(d.abs() / out_tol.clamp(min=1e-12)).nan_to_num(9e9).max().item():.3g} of the tolerance"
        dl = (got["lse"].double() - lse).abs()
        assert ((dl <= lse_tol) | (got["lse"].double() == lse) | (torch.isnan(lse) & torch.isnan(got["lse"]))).all()


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("dim", [64, 96, 128])
@pytest.mark.parametrize("new,lens", [([1], [1]), ([1], [65]), ([1, 1, 1], [16, 17, 1000]), ([2, 1, 5], [2, 300, 64]), ([130], [130]), ([33, 1, 300], [500, 129, 300])])
def test_attention_types_and_lengths(gorio, dtype, dim, new, lens):
    Case(new, lens, dim=dim, dtype=dtype, seed=dim).check(gorio)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 1), (3, 3), (10, 2), (14, 2), (32, 2), (40, 1), (9, 3)])
@pytest.mark.parametrize("new", [1, 3, 70, 900])
def test_attention_head_layouts(gorio, heads, kv_heads, new):
    Case([new, 1], [max(new, 211), 90], heads=heads, kv_heads=kv_heads, dim=128, seed=heads).check(gorio)


@pytest.mark.parametrize("page", [8, 16, 24, 48, 64, 128, 256])
@pytest.mark.parametrize("layout", ["heads", "tokens", "joint"])
@pytest.mark.parametrize("new", [1, 150])
def test_attention_pages_and_strides(gorio, page, layout, new):
    Case([new, 1], [777, 40], page=page, layout=layout, dim=96 if page == 48 else 64, seed=page).check(gorio)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [0, 1, 5, 64, 200])
@pytest.mark.parametrize("softcap,slopes", [(0.0, False), (5.0, False), (0.0, True), (30.0, True)])
@pytest.mark.parametrize("new", [[1, 1, 1], [40, 1, 260]])
def test_attention_masks_and_scores(gorio, causal, window, softcap, slopes, new):
    Case(new, [300, 150, 430], dim=128 if softcap else 64, causal=causal, window=window, softcap=softcap, slopes=slopes, seed=window, freed=window > 0).check(gorio)


def test_attention_rows_without_keys(gorio):
    # no keys at all; fewer keys than new tokens (the first queries stand before the first key)
    for causal in (True, False):
        for new in ([1, 2, 1], [5, 9, 3], [40, 300, 7]):
            c = Case(new, [0, 2, 0], causal=causal)
            got = c.check(gorio)
            assert (got["out"][:new[0]] == 0).all() and (got["lse"][:new[0]] == -math.inf).all()
    # a request without new tokens between others; no request at all
    Case([1, 0, 1], [40, 30, 20]).check(gorio)
    Case([0, 0, 70], [40, 30, 100]).check(gorio)
    c = Case([0, 0], [4, 5])
    assert c.run(gorio)["out"].shape == (0, 8, 64)


@pytest.mark.parametrize("new", [[4], [1], [150]])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_attention_values_that_are_not_finite_reach_only_who_sees_them(gorio, new, bad):
    c = Case(new, [200], dim=64, heads=8, kv_heads=2)
    page = c.tables[0, 198 // 16].item()
    c.vp[page, :, 198 % 16, 3] = bad                           # all but the last two tokens' queries do not see it
    got = c.check(gorio)
    assert torch.isfinite(got["out"][: max(0, new[0] - 2)]).all()
    assert not torch.isfinite(got["out"][-1, :, 3]).any() and torch.isfinite(got["out"][-1, :, 4]).all()
    c = Case(new, [200], dim=64, heads=8, kv_heads=2)
    c.kp[page, :, 198 % 16, 3] = math.nan                      # a score that is not a number
    got = c.run(gorio)
    assert torch.isfinite(got["out"][: max(0, new[0] - 2)]).all() and torch.isnan(got["out"][-1]).all()


@pytest.mark.parametrize("new", [1, 100])
def test_attention_extreme_scores(gorio, new):
    # weights that all but vanish beside one key's, and scores far from 0
    Case([new], [500], sharp=60.0, dim=128, heads=16, kv_heads=4).check(gorio)
    c = Case([new], [500], dim=128, heads=16, kv_heads=4)
    c.q.zero_()                                                # even weights: the mean of the values
    c.check(gorio)


def test_attention_long_cache_in_parts(gorio):
    """One request over a long cache is cut between all blocks; more requests than threads of a block."""
    Case([1], [40000], dim=128, heads=8, kv_heads=2, page=64).check(gorio)
    Case([1, 1], [9000, 3], dim=64, heads=5, kv_heads=1).check(gorio)
    Case([60], [20000], dim=64, heads=8, kv_heads=1, page=64).check(gorio)
    Case([150], [20000], dim=64, heads=8, kv_heads=1, page=64).check(gorio)           # units of both sizes, cut often
    Case([150], [9000], dim=128, heads=6, kv_heads=1).check(gorio)
    Case([30] * 7, [9000, 100, 300, 5, 2000, 700, 30], dim=128, heads=6, kv_heads=2).check(gorio)
    Case([300, 40, 7], [4000, 900, 2500], dim=96, heads=4, kv_heads=2).check(gorio)
    rng = random.Random(5)
    Case([1] * 1500, [rng.randint(0, 40) for _ in range(1500)], dim=64, heads=2, kv_heads=1).check(gorio)
    Case([rng.randint(0, 3) for _ in range(700)], [rng.randint(0, 90) for _ in range(700)], dim=64, heads=2, kv_heads=1).check(gorio)


def test_attention_of_many_requests_with_chunks(gorio):
    """More requests than threads of a block, most of them of more rows than the single-token form takes."""
    rng = random.Random(6)
    Case([rng.randint(0, 20) for _ in range(500)], [rng.randint(0, 150) for _ in range(500)], dim=64, heads=2, kv_heads=1, page=8).check(gorio)
    Case([3] * 40 + [200], [200] * 41, dim=128, heads=8, kv_heads=1, causal=False).check(gorio)


@pytest.mark.parametrize("new", [1, 50, 250])
def test_attention_scale(gorio, new):
    c = Case([new], [300], dim=64, heads=4, kv_heads=2)
    got = c.run(gorio, scale=0.03)
    out, lse, out_tol, lse_tol = plain_attention(c.q, c.kp, c.vp, c.tables, c.lengths, c.starts, scale=0.03)
    assert ((got["out"].double() - out).abs() <= out_tol).all() and ((got["lse"].double() - lse).abs() <= lse_tol).all()
    with pytest.raises(gorio.GorioError):
        c.run(gorio, scale=0.0)
    with pytest.raises(gorio.GorioError):
        c.run(gorio, window=-1)
    with pytest.raises(gorio.GorioError):
        gorio.paged_attention(c.q[:, :3], c.kp, c.vp, c.tables, c.lengths, c.starts, new)
    with pytest.raises(gorio.GorioError):
        gorio.paged_attention(c.q, c.kp, c.vp.half(), c.tables, c.lengths, c.starts, new)
    with pytest.raises(gorio.GorioError):
        gorio.paged_attention(c.q, c.kp, c.vp, c.tables, c.lengths, c.starts[:1], new)
    with pytest.raises(gorio.GorioError):
        gorio.paged_attention(c.q, c.kp, c.vp, c.tables, c.lengths, c.starts, new, workspace=torch.zeros(100, dtype=torch.uint8, device="cuda"))
    with pytest.raises(gorio.GorioError):
        gorio.cache_store(c.q, c.q, c.kp, c.vp, torch.zeros(c.q.shape[0], dtype=torch.int64, device="cuda"))


def test_attention_offsets_past_32_bits(gorio):
    """The pages in use lie behind the 2^31st element (and the 2^32nd byte) of the cache."""
    spare = (1 << 31) // (2 * 64 * 128) + 8
    for new in (1, 250):
        Case([new, 1], [500, 300], dim=128, heads=4, kv_heads=2, page=64, spare=spare).check(gorio)
        torch.cuda.empty_cache()


@pytest.mark.parametrize("new", [40, 140])
def test_attention_table_entries_outside_the_cache_read_as_zeros(gorio, new):
    c = Case([1, new], [100, 200])
    want = None
    for bad in (-1, 1 << 30):
        c.tables[0, 2] = bad
        c.tables[1, 3] = bad
        got = c.run(gorio)
        assert torch.isfinite(got["out"]).all()
        assert want is None or torch.equal(got["out"], want)
        want = got["out"]
    # lengths and starts that promise more than there is
    c.lengths[0] = 1 << 30
    c.starts[2] = 1 << 30
    c.run(gorio)
    c.lengths[0] = -5
    c.starts[0] = -9
    c.run(gorio)
    torch.cuda.synchronize()


@pytest.mark.parametrize("new", [30, 130])
def test_attention_does_not_change_between_calls_streams_and_graphs(gorio, new):
    c = Case([1, new, 1], [5000, 900, 77], dim=128, heads=8, kv_heads=2)
    first = c.run(gorio)
    for _ in range(3):
        again = c.run(gorio)
        assert torch.equal(first["out"], again["out"]) and torch.equal(first["lse"], again["lse"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = c.run(gorio, stream=side)
    side.synchronize()
    assert torch.equal(first["out"], other["out"])
    graph = torch.cuda.CUDAGraph()
    ws = gorio.attention_workspace()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        held = c.run(gorio, workspace=ws)
        fresh = c.run(gorio)                                   # a workspace of the graph's own
    for _ in range(2):
        held["out"].zero_(), fresh["out"].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(first["out"], held["out"]) and torch.equal(first["out"], fresh["out"])
    c.compare(first)


def test_attention_max_new_is_a_hint(gorio):
    c = Case([1, 130], [300, 200], dim=128)
    for max_new in (0, 1, 130, 5000):
        c.check(gorio, max_new=max_new)


def test_attention_check_reports_a_wait_that_ran_out(gorio):
    c = Case([140, 1], [160, 200])
    ws = gorio.attention_workspace()
    c.run(gorio, workspace=ws)
    gorio.attention_check(ws)
    gorio.attention_check()
    ws[(1 << 16) - 4] = 1                                      # what a kernel leaves when a wait passes its limit
    with pytest.raises(gorio.GorioError) as e:
        gorio.attention_check(ws)
    assert e.value.status == 5
    gorio.attention_check(ws)
    c.compare(c.run(gorio, workspace=ws))
    assert (ws[: 1 << 16] == 0).all()


def test_attention_into_a_given_tensor(gorio):
    c = Case([5, 1], [300, 200], heads=4, dim=64)
    wide = torch.zeros((6, 4, 72), dtype=BF16, device="cuda")
    got = c.check(gorio, out=wide[..., :64])
    assert got["out"].data_ptr() == wide.data_ptr() and (wide[..., 64:] == 0).all()


def test_tables_store_and_attention_together(gorio):
    """Tokens that go through tables and store give what the same tokens give in one step."""
    g = torch.Generator(device="cuda").manual_seed(3)
    heads, kv, dim, page, total = 4, 2, 64, 16, 45
    q = torch.randn((total, heads, dim), generator=g, device="cuda").to(BF16)
    kv_new = torch.randn((total, 2, kv, dim), generator=g, device="cuda").to(BF16)

    def serve(steps):
        kp = torch.full((8, kv, page, dim), math.nan, dtype=BF16, device="cuda")
        vp = kp.clone()
        tables = torch.full((1, 4), -1, dtype=torch.int32, device="cuda")
        lengths, count, free = _i32([0]), _i32([8]), _i32([3, 1, 4, 0, 5, 2, 7, 6])
        outs, at = [], 0
        for n in steps:
            p = gorio.page_tables(lengths, _i32([n]), tables, free, count, page, n)
            lengths, count = p["lengths"], p["free_count"]
            gorio.cache_store(kv_new[at:at + n, 0], kv_new[at:at + n, 1], kp, vp, p["slots"])
            outs.append(gorio.paged_attention(q[at:at + n], kp, vp, tables, lengths, p["starts"], n)["out"])
            at += n
        return torch.cat(outs)
    whole = serve([total])
    pieces = serve([20, 1, 1, 13, 1, 9])
    # both are within the tolerance of the same exact result
    dense_k = kv_new[:, 0].transpose(0, 1).reshape(1, kv, total, dim)
    pad = torch.zeros((1, kv, 48 - total, dim), dtype=BF16, device="cuda")
    out, _, tol, _ = plain_attention(q, torch.cat([dense_k, pad], 2), torch.cat([kv_new[:, 1].transpose(0, 1).reshape(1, kv, total, dim), pad], 2),
                                     _i32([[0]]), _i32([total]), _i32([0, total]))
    assert ((whole.double() - out).abs() <= tol).all() and ((pieces.double() - out).abs() <= tol).all()


def test_example_from_a_search_to_attention(gorio):
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "retrieve_and_attend.py")
    spec = importlib.util.spec_from_file_location("retrieve_and_attend", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.main(questions=9, steps=2, heads=8, kv_heads=2)
    assert r["served"].tolist() == [1] * 9
    out, lse, out_tol, lse_tol = plain_attention(r["q"], r["key_pages"], r["value_pages"], r["tables"], r["lengths"], r["starts"])
    assert ((r["out"].double() - out).abs() <= out_tol).all() and ((r["lse"].double() - lse).abs() <= lse_tol).all()
